// C ABI of the prompt side (include/delta_extend.h): argument checks, the cut of a call into tiles
// and splits, the workspace layout, and the launches.
#include <math.h>

#include <algorithm>

#include "api_common.h"
#include "extend.h"
#include "runs_api.h"

namespace delta {

// Most pieces that a call's keys are cut into, and most (row, query head) parts of outputs that it
// keeps (68 MB at head size 128): with the second a call's workspace grows with its rows and nothing
// else, so that one sized for the most rows serves every smaller call.
constexpr int kMostSplits = 32, kMostParts = 1 << 17;
// Which kernel, and into how many pieces the keys are cut.  The host knows no run but the longest, so
// it takes the rows for runs of that length and single tokens.
//
// A workgroup of the many-row kernel takes 64 keys in 2.2 us when its 256 rows are full (a tile of a
// single token about a quarter), one of the few-row kernel 128 keys in 1.2 us while it has a CU to
// itself.  Keys are cut until the workgroups fill the 256 CUs (more pieces only add partial outputs
// and their join, fewer leave CUs idle), and the kernel is the one whose last CU is done first; four
// units of 1.2 us are what the many-row kernel's start and its LDS exchange cost more.
// Measured on MI355X, us, few- and many-row kernel with this number of pieces, 32/8 heads, one
// sequence: prompts of 128 tokens 6.9 and 12.2, 512 13.4 and 24, 1024 33 and 36, 2048 85 and 73, 4096
// 303 and 168; 256 tokens behind a prefix of 7936 93 and 55; eight prompts of 256 35 and 20; eight
// times 16 tokens at 4096 37 and 36.
ExtendPlan plan_extend(const delta_shape_t* s, int n_rows, int max_new) {
  constexpr int kCus = 256, kFewestKeys = 256, kStart = 4;
  const int G = s->n_q_heads / s->n_kv_heads;
  const double keys = s->max_seq_len;
  const int spare = std::max(0, n_rows - s->batch);   // rows beyond one per sequence
  const double runs = max_new > 1 ? std::min<double>(s->batch, std::max(1.0, round((double)spare / (max_new - 1)))) : 0;
  struct Cut {
    double cost;
    int splits;
  };
  auto cut = [&](int rows, double light, double keys_per_unit) {
    const double tiles = runs * ceil((double)max_new * G / rows) + light * (s->batch - runs);
    const double wgs = std::max(1.0, tiles * s->n_kv_heads);
    const double parts = (double)kMostParts / std::max<int64_t>(1, (int64_t)n_rows * s->n_q_heads);
    const int splits = (int)std::max(1.0, std::min({kCus / wgs, (double)kMostSplits, keys / kFewestKeys, parts}));
    return Cut{keys / keys_per_unit / splits * std::max(1.0, wgs * splits / kCus), splits};
  };
  const Cut few = cut(32, 1.0, 128), many = cut(256, 0.25, 32);
  // the grid: every run ends in a partial tile, so at most one tile per run more than whole ones
  auto tiles_of = [&](int rows) {
    const int64_t by_run = (int64_t)s->batch * (((int64_t)max_new * G + rows - 1) / rows);
    const int64_t by_row = (int64_t)n_rows * G / rows + std::min(s->batch, n_rows);
    return (int)std::min(by_run, by_row);
  };
  // (what the few-row kernel's smaller tiles would make too many goes to the other, whose tiles never
  // get fewer with more rows or longer runs: a call that is taken has no smaller one that is refused)
  const bool is_few =
      ((int64_t)max_new * G <= 32 || few.cost <= many.cost + kStart) && tiles_of(32) <= kMostTiles;
  ExtendPlan p;
  p.rows = is_few ? 32 : 256;
  p.tiles = tiles_of(p.rows);
  const int n = is_few ? few.splits : many.splits;
  p.split_keys = ceil_div(ceil_div(s->max_seq_len, n), kFewestKeys) * kFewestKeys;
  p.n_split = ceil_div(s->max_seq_len, p.split_keys);
  return p;
}

}  // namespace delta

namespace {

using namespace delta;

struct ExtendLayout {
  ExtendPlan plan;
  int n_rows = 0;   // rows that can belong to a run
  size_t status = 0, part_ml = 0, part_n = 0, part_o = 0, total = 0;
};

// Bytes of `rows` (row, query head) pairs in `parts` parts.
size_t lay_out(size_t rows, size_t parts, int head_dim, ExtendLayout* L) {
  size_t off = 0;
  L->status = off;  off = align_up(off + sizeof(uint32_t));
  L->part_ml = off; off = align_up(off + sizeof(float) * 2 * parts);
  L->part_n = off;  off = align_up(off + sizeof(int32_t) * rows);
  L->part_o = off;  off = align_up(off + sizeof(float) * head_dim * parts);
  return off;
}

int extend_layout(const delta_shape_t* s, int32_t n_rows, int32_t max_new, ExtendLayout* L) {
  int rc = check_shape(s);
  if (rc) return rc;
  if (n_rows < 0 || max_new < 0 || max_new > n_rows) return DELTA_ERR_INVALID_ARG;
  if ((int64_t)n_rows * s->n_q_heads > (1 << 28) || s->max_seq_len > kMostKeys) return DELTA_ERR_UNSUPPORTED;
  L->n_rows = (int)std::min<int64_t>(n_rows, (int64_t)s->batch * max_new);
  L->plan = plan_extend(s, L->n_rows, max_new);
  if (L->plan.tiles > kMostTiles) return DELTA_ERR_UNSUPPORTED;
  const size_t rows = (size_t)L->n_rows * s->n_q_heads;
  if (L->plan.n_split > 1) L->total = lay_out(rows, L->plan.n_split * rows, s->head_dim, L);
  else L->total = lay_out(0, 0, s->head_dim, L);
  return DELTA_OK;
}

}  // namespace

#pragma GCC visibility push(default)
extern "C" {

int delta_rope_append(const delta_shape_t* shape, const delta_kv_t* kv, const delta_rope_t* rope,
                      int32_t n_rows, const int32_t* row_offsets, const void* q,
                      int64_t q_row_stride, const void* k, int64_t k_row_stride, const void* v,
                      int64_t v_row_stride, void* q_out, void* stream) {
  RopeAppendArgs a{};
  const int rc = append_args(shape, kv, rope, n_rows, row_offsets, q, q_row_stride, k, k_row_stride, v, v_row_stride,
                             q_out, &a);
  if (rc || n_rows == 0) return rc;
  return hip_rc(launch_rope_append(shape->head_dim, is_e4m3(kv), a, static_cast<hipStream_t>(stream)));
}

int delta_extend_workspace_bytes(const delta_shape_t* shape, int32_t n_rows, int32_t max_new, size_t* out) {
  if (!out) return DELTA_ERR_INVALID_ARG;
  ExtendLayout L;
  int rc = extend_layout(shape, n_rows, max_new, &L);
  if (rc) return rc;
  const size_t rows = (size_t)L.n_rows * shape->n_q_heads, most = kMostParts;
  *out = lay_out(std::min(rows, most), std::min(kMostSplits * rows, most), shape->head_dim, &L);
  return DELTA_OK;
}

int delta_extend_attn(const delta_shape_t* shape, const delta_kv_t* kv, int32_t n_rows,
                      int32_t max_new, const int32_t* row_offsets, const void* q, void* out,
                      void* ws, size_t ws_bytes, void* stream) {
  ExtendLayout L;
  int rc = extend_layout(shape, n_rows, max_new, &L);
  if (rc) return rc;
  if ((rc = check_kv(kv))) return rc;
  if ((rc = check_runs(shape, n_rows, row_offsets))) return rc;
  if (!row_offsets && max_new < 1) return DELTA_ERR_INVALID_ARG;
  if (!ws) return DELTA_ERR_INVALID_ARG;
  if (ws_bytes < L.total) return DELTA_ERR_WORKSPACE;
  if (n_rows == 0 || max_new == 0) return DELTA_OK;
  if (!q || !out) return DELTA_ERR_INVALID_ARG;
  for (const void* p : {q, static_cast<const void*>(out), kv->k_cache, kv->v_cache})
    if (!aligned(p, 16)) return DELTA_ERR_INVALID_ARG;
  if (!aligned(ws, 256)) return DELTA_ERR_INVALID_ARG;
  char* w = static_cast<char*>(ws);
  ExtendArgs a = extend_args(shape, kv, L.n_rows, row_offsets, q, out);
  a.part_ml = reinterpret_cast<float*>(w + L.part_ml);
  a.part_o = reinterpret_cast<float*>(w + L.part_o);
  a.part_n = reinterpret_cast<int32_t*>(w + L.part_n);
  a.n_split = L.plan.n_split;
  a.split_keys = L.plan.split_keys;
  a.status = reinterpret_cast<uint32_t*>(w + L.status);
  return hip_rc(launch_extend(L.plan, shape->head_dim, is_e4m3(kv), a, static_cast<hipStream_t>(stream)));
}

}  // extern "C"
#pragma GCC visibility pop
