// C ABI of a round of drafted tokens (include/delta_drafts.h): argument checks, the cut of attention calls
// into tiles and pieces, workspace layouts, and the launches.
#include <math.h>

#include <algorithm>

#include "api_common.h"
#include "drafts.h"
#include "runs_api.h"

namespace delta {

namespace {

constexpr int kCus = 256;

// Most tiles of a call, whatever its longest run: every run ends in a partial tile, so at most one tile per run more
// than whole ones.
int64_t most_tiles(const delta_shape_t* s, int n_rows, int tile_rows) {
  return (int64_t)n_rows * (s->n_q_heads / s->n_kv_heads) / tile_rows + std::min(s->batch, n_rows);
}

// Units of a tile of the longest sequence, most groups that fill the GPU, and most that a call with so many tiles has.
int64_t most_units(const delta_shape_t* s) { return kTileUnits + kMostUnits64 * ((int64_t)s->max_seq_len / 64 + 4); }
int64_t full_groups(const delta_shape_t* s) { return std::max(1, kCus / s->n_kv_heads); }
int64_t most_groups(const delta_shape_t* s, int64_t tiles) {
  return std::min(full_groups(s), tiles * (1 + most_units(s) / kLeastUnits) + 1);
}

}  // namespace

// Tiles of 32 rows, where a group's workgroups have up to six of their blocks of 128 keys to walk: then what a tile
// costs before and after its walk decides, and four waves start and end sooner than eight.  Measured on MI355X, us,
// tiles of 32 and 256 rows: 28/4 heads, a tree of 16 behind 8192 tokens (4 blocks) 20.5 and 23.2, 32768 (16) 44 and
// 34; 32/8 heads, 64 behind 2048 (4) 20.1 and 26.7; 16 sequences of 4K-16K, 16 rows each 232 and 153.
TreePlan plan_tree(const delta_shape_t* s, int n_rows, int max_new) {
  const int G = s->n_q_heads / s->n_kv_heads;
  const int64_t full = full_groups(s);
  auto tiles_of = [&](int tile_rows) {
    const int64_t by_run = (int64_t)s->batch * (((int64_t)max_new * G + tile_rows - 1) / tile_rows);
    return std::min(by_run, most_tiles(s, n_rows, tile_rows));
  };
  const bool few = (int64_t)max_new * G <= 32 ||
                   (s->batch <= kCutBatch && tiles_of(32) * ((int64_t)s->max_seq_len / 128 + 1) <= 6 * full);
  TreePlan p;
  p.rows = few ? 32 : 256;
  p.tiles = (int)tiles_of(p.rows);
  const int64_t tiles = most_tiles(s, n_rows, p.rows);
  // (short sequences: joining parts takes 3 us, as long as walking two or three of these blocks)
  if (s->max_seq_len <= 768 || s->batch > kCutBatch || tiles * most_units(s) >= 1 << 30) return p;
  // A group's units, with pieces of tiles and with equal parts of all of them, by the bound of the lengths: the
  // first where what they are longer is less than the second tile that most equal parts touch.
  const int64_t blocks = tiles * 4 * ((int64_t)s->max_seq_len / 64 + 4);
  const int64_t equal = std::max<int64_t>(kLeastUnits, (blocks + kTileUnits * tiles) / full);
  p.pieces = tiles < full && std::max<int64_t>(kLeastUnits, blocks / (full - tiles)) <= equal + kTileUnits;
  p.workgroups = s->n_kv_heads * (int)most_groups(s, tiles);
  return p;
}

}  // namespace delta

namespace {

using namespace delta;

// Runs of trees: rows of calls that need no cache.
int check_drafts(int32_t batch, int32_t n_rows, int32_t max_new, const int32_t* row_offsets) {
  if (batch < 1 || n_rows < 0 || max_new < 0 || max_new > n_rows) return DELTA_ERR_INVALID_ARG;
  if (!row_offsets && (n_rows != batch || max_new < 1)) return DELTA_ERR_INVALID_ARG;
  if (batch > 65535 || n_rows >= 1 << 24 || max_new > kMostDrafts) return DELTA_ERR_UNSUPPORTED;
  return DELTA_OK;
}

struct TreeLayout {
  TreePlan plan;
  int n_rows = 0;   // rows that can belong to a run
  size_t status = 0, part_ml = 0, part_n = 0, part_o = 0, total = 0;
};

// Bytes of a call's workspace; every workgroup of a shared call has room for two parts of a tile.
size_t lay_out(const delta_shape_t* s, int n_rows, const TreePlan& p, TreeLayout* L) {
  const size_t parts = 2 * (size_t)p.workgroups * p.rows, rows = p.workgroups ? (size_t)n_rows * s->n_q_heads : 0;
  size_t off = 0;
  L->status = off;  off = align_up(off + sizeof(uint32_t));
  L->part_ml = off; off = align_up(off + sizeof(float) * 2 * parts);
  L->part_n = off;  off = align_up(off + sizeof(int32_t) * rows);
  L->part_o = off;  off = align_up(off + sizeof(float) * s->head_dim * parts);
  return off;
}

int tree_layout(const delta_shape_t* s, int32_t n_rows, int32_t max_new, TreeLayout* L) {
  int rc = check_shape(s);
  if (rc) return rc;
  if (n_rows < 0 || max_new < 0 || max_new > n_rows) return DELTA_ERR_INVALID_ARG;
  if ((int64_t)n_rows * s->n_q_heads > (1 << 28) || s->max_seq_len > kMostKeys || max_new > kMostDrafts)
    return DELTA_ERR_UNSUPPORTED;
  L->n_rows = (int)std::min<int64_t>(n_rows, (int64_t)s->batch * max_new);
  L->plan = plan_tree(s, L->n_rows, max_new);
  if (L->plan.tiles > kMostTiles) return DELTA_ERR_UNSUPPORTED;
  L->total = lay_out(s, L->n_rows, L->plan, L);
  return DELTA_OK;
}

}  // namespace

#pragma GCC visibility push(default)
extern "C" {

int delta_norm_rope_append(const delta_shape_t* shape, const delta_kv_t* kv, const delta_norm_t* norm,
                           const delta_rope_t* rope, int32_t n_rows, const int32_t* row_offsets, const void* q,
                           int64_t q_row_stride, const void* k, int64_t k_row_stride, const void* v,
                           int64_t v_row_stride, void* q_out, void* stream) {
  if (!norm || (norm->weight_type != DELTA_NORM_BF16 && norm->weight_type != DELTA_NORM_F32) || !(norm->eps >= 0.f) ||
      isinf(norm->eps) || !aligned(norm->q_weight, 16) || !aligned(norm->k_weight, 16))
    return DELTA_ERR_INVALID_ARG;
  RopeAppendArgs a{};
  const int rc = append_args(shape, kv, rope, n_rows, row_offsets, q, q_row_stride, k, k_row_stride, v, v_row_stride,
                             q_out, &a);
  if (rc || n_rows == 0) return rc;
  const HeadNorm h{norm->q_weight, norm->k_weight, norm->weight_type == DELTA_NORM_F32, norm->eps};
  return hip_rc(launch_norm_rope_append(shape->head_dim, is_e4m3(kv), a, h, static_cast<hipStream_t>(stream)));
}

int delta_tree_layout(const delta_shape_t* shape, const int32_t* seq_lens, int32_t n_rows, int32_t max_new,
                      const int32_t* row_offsets, const int32_t* parents, int32_t* positions, uint32_t* masks,
                      int32_t mask_words, void* stream) {
  if (!shape) return DELTA_ERR_INVALID_ARG;
  int rc = check_drafts(shape->batch, n_rows, max_new, row_offsets);
  if (rc) return rc;
  if (masks && (mask_words < 1 || mask_words < ceil_div(max_new, 32))) return DELTA_ERR_INVALID_ARG;
  if (n_rows == 0 || max_new == 0) return DELTA_OK;
  if (!parents || (!positions && !masks) || (positions && !seq_lens)) return DELTA_ERR_INVALID_ARG;
  TreeLayoutArgs a{};
  a.runs = Runs{row_offsets, seq_lens, nullptr, n_rows, shape->batch, 0};
  a.parents = parents;
  a.positions = positions;
  a.masks = masks;
  a.mask_words = mask_words;
  a.max_new = max_new;
  return hip_rc(launch_tree_layout(a, static_cast<hipStream_t>(stream)));
}

int delta_tree_workspace_bytes(const delta_shape_t* shape, int32_t n_rows, int32_t max_new, size_t* out) {
  if (!out) return DELTA_ERR_INVALID_ARG;
  TreeLayout L;
  int rc = tree_layout(shape, n_rows, max_new, &L);
  if (rc) return rc;
  // of either tile: a smaller call may take the smaller one, of which there are more
  *out = L.total;
  TreePlan p = L.plan;
  for (p.rows = 32; p.rows <= L.plan.rows; p.rows *= 8) {
    p.workgroups = shape->n_kv_heads * (int)most_groups(shape, most_tiles(shape, L.n_rows, p.rows));
    *out = std::max(*out, lay_out(shape, L.n_rows, p, &L));
  }
  return DELTA_OK;
}

int delta_tree_attn(const delta_shape_t* shape, const delta_kv_t* kv, int32_t n_rows, int32_t max_new,
                    const int32_t* row_offsets, const uint32_t* masks, int32_t mask_words, const void* q,
                    void* out, void* ws, size_t ws_bytes, void* stream) {
  TreeLayout L;
  int rc = tree_layout(shape, n_rows, max_new, &L);
  if (rc) return rc;
  if ((rc = check_kv(kv))) return rc;
  if ((rc = check_runs(shape, n_rows, row_offsets))) return rc;
  if (!row_offsets && max_new < 1) return DELTA_ERR_INVALID_ARG;
  if (mask_words < 1 || mask_words < ceil_div(max_new, 32)) return DELTA_ERR_INVALID_ARG;
  if (!ws) return DELTA_ERR_INVALID_ARG;
  if (ws_bytes < L.total) return DELTA_ERR_WORKSPACE;
  if (n_rows == 0 || max_new == 0) return DELTA_OK;
  if (!q || !out || !masks) return DELTA_ERR_INVALID_ARG;
  for (const void* p : {q, static_cast<const void*>(out), kv->k_cache, kv->v_cache})
    if (!aligned(p, 16)) return DELTA_ERR_INVALID_ARG;
  if (!aligned(ws, 256)) return DELTA_ERR_INVALID_ARG;
  char* w = static_cast<char*>(ws);
  ExtendArgs a = extend_args(shape, kv, L.n_rows, row_offsets, q, out);
  a.part_ml = reinterpret_cast<float*>(w + L.part_ml);
  a.part_o = reinterpret_cast<float*>(w + L.part_o);
  a.part_n = reinterpret_cast<int32_t*>(w + L.part_n);
  a.status = reinterpret_cast<uint32_t*>(w + L.status);
  a.masks = masks;
  a.mask_words = mask_words;
  return hip_rc(launch_tree_attn(L.plan, shape->head_dim, is_e4m3(kv), a, static_cast<hipStream_t>(stream)));
}

int delta_verify_workspace_bytes(int32_t batch, int32_t vocab, size_t* out) {
  if (!out || batch < 1 || vocab < 1) return DELTA_ERR_INVALID_ARG;
  if (batch > 65535 || vocab > kMostVocab) return DELTA_ERR_UNSUPPORTED;
  *out = sizeof(VerifyState) * (size_t)batch;
  return DELTA_OK;
}

int delta_verify_drafts(int32_t batch, int32_t n_rows, int32_t max_new, const int32_t* row_offsets, int32_t vocab,
                        const float* target, int64_t target_row_stride, const float* draft,
                        int64_t draft_row_stride, const int32_t* tokens, const int32_t* parents,
                        const float* uniform, int32_t* path, int32_t* n_path, int32_t* next, void* ws,
                        size_t ws_bytes, void* stream) {
  int rc = check_drafts(batch, n_rows, max_new, row_offsets);
  if (rc) return rc;
  if (max_new < 1 || vocab < 1 || target_row_stride < vocab || (draft && draft_row_stride < vocab))
    return DELTA_ERR_INVALID_ARG;
  if (vocab > kMostVocab) return DELTA_ERR_UNSUPPORTED;
  if (!target || !tokens || !parents || !uniform || !path || !n_path || !next || !ws || !aligned(ws, 256))
    return DELTA_ERR_INVALID_ARG;
  if (ws_bytes < sizeof(VerifyState) * (size_t)batch) return DELTA_ERR_WORKSPACE;
  VerifyArgs a{};
  a.runs = Runs{row_offsets, nullptr, nullptr, n_rows, batch, 0};
  a.target = target;
  a.draft = draft;
  a.target_stride = target_row_stride;
  a.draft_stride = draft_row_stride;
  a.tokens = tokens;
  a.parents = parents;
  a.uniform = uniform;
  a.path = path;
  a.n_path = n_path;
  a.next = next;
  a.state = static_cast<VerifyState*>(ws);
  a.vocab = vocab;
  a.max_new = max_new;
  // one round of loads a wave; two where that would be more workgroups than fit the GPU at once
  a.part = kMostPart / 2;
  a.n_pieces = ceil_div(vocab, kVerifyWaves * a.part);
  if (a.n_pieces > kMostPieces || (int64_t)a.n_pieces * batch > 1536) {
    a.part = kMostPart;
    a.n_pieces = ceil_div(vocab, kVerifyWaves * a.part);
  }
  return hip_rc(launch_verify(a, static_cast<hipStream_t>(stream)));
}

int delta_cache_compact(const delta_shape_t* shape, int32_t n_layers, const delta_kv_t* kv, int32_t n_rows,
                        int32_t max_new, const int32_t* row_offsets, const int32_t* path, const int32_t* n_path,
                        int32_t* new_lens, void* stream) {
  int rc = check_shape(shape);
  if (rc) return rc;
  if (n_layers < 1 || !kv) return DELTA_ERR_INVALID_ARG;
  for (int i = 0; i < n_layers; ++i) {
    if ((rc = check_kv(kv + i))) return rc;
    if (kv[i].seq_lens != kv[0].seq_lens || !aligned(kv[i].k_cache, 16) || !aligned(kv[i].v_cache, 16))
      return DELTA_ERR_INVALID_ARG;
    // (a cache that is named twice would be moved twice at once)
    if (kv[i].k_cache == kv[i].v_cache) return DELTA_ERR_INVALID_ARG;
    for (int j = 0; j < i; ++j)
      for (const void* p : {kv[i].k_cache, kv[i].v_cache})
        if (p == kv[j].k_cache || p == kv[j].v_cache) return DELTA_ERR_INVALID_ARG;
  }
  if ((rc = check_drafts(shape->batch, n_rows, max_new, row_offsets))) return rc;
  if (max_new < 1 || !path || !n_path) return DELTA_ERR_INVALID_ARG;
  const bool in_place = new_lens && new_lens == kv[0].seq_lens;
  CompactArgs a{};
  a.runs = Runs{row_offsets, kv[0].seq_lens, nullptr, n_rows, shape->batch, shape->max_pages_per_seq};
  a.path = path;
  a.n_path = n_path;
  a.max_new = max_new;
  a.n_kv_heads = shape->n_kv_heads;
  a.head_dim = shape->head_dim;
  for (int first = 0; first < n_layers; first += kLayersPerLaunch) {
    a.n_layers = std::min(kLayersPerLaunch, n_layers - first);
    a.new_lens = first || in_place ? nullptr : new_lens;
    a.e4m3 = 0;
    for (int i = 0; i < a.n_layers; ++i) {
      const delta_kv_t& l = kv[first + i];
      // (the cache descriptor is shared with the calls that only read it)
      a.layers[i] = CompactLayer{static_cast<uint8_t*>(const_cast<void*>(l.k_cache)),
                                 static_cast<uint8_t*>(const_cast<void*>(l.v_cache)), l.page_table, l.n_pages};
      if (is_e4m3(&l)) a.e4m3 |= (uint64_t)1 << i;
    }
    if ((rc = hip_rc(launch_compact(a, static_cast<hipStream_t>(stream))))) return rc;
  }
  if (in_place) {
    a.new_lens = new_lens;
    rc = hip_rc(launch_compact_lens(a, static_cast<hipStream_t>(stream)));
  }
  return rc;
}

}  // extern "C"
#pragma GCC visibility pop
