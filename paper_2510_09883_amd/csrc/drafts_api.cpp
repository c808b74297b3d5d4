// C ABI of a round of drafted tokens (include/delta_drafts.h): argument checks, the cut of attention calls
// into tiles and pieces, workspace layouts, and the launches.
#include <math.h>

#include <algorithm>

#include "api_common.h"
#include "drafts.h"
#include "runs_api.h"

namespace delta {

ExtendPlan plan_tree(const delta_shape_t* s, int n_rows, int max_new) { return plan_extend(s, n_rows, max_new); }

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

int tree_layout(const delta_shape_t* s, int32_t n_rows, int32_t max_new, ExtendLayout* L) {
  int rc = check_shape(s);
  if (rc) return rc;
  if (n_rows < 0 || max_new < 0 || max_new > n_rows) return DELTA_ERR_INVALID_ARG;
  if ((int64_t)n_rows * s->n_q_heads > (1 << 28) || s->max_seq_len > kMostKeys || max_new > kMostDrafts)
    return DELTA_ERR_UNSUPPORTED;
  L->n_rows = (int)std::min<int64_t>(n_rows, (int64_t)s->batch * max_new);
  L->plan = plan_tree(s, L->n_rows, max_new);
  if (L->plan.tiles > kMostTiles) return DELTA_ERR_UNSUPPORTED;
  const size_t rows = (size_t)L->n_rows * s->n_q_heads;
  if (L->plan.n_split > 1) L->total = lay_out(rows, L->plan.n_split * rows, s->head_dim, L);
  else L->total = lay_out(0, 0, s->head_dim, L);
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
  ExtendLayout L;
  int rc = tree_layout(shape, n_rows, max_new, &L);
  if (rc) return rc;
  const size_t rows = (size_t)L.n_rows * shape->n_q_heads, most = kMostParts;
  *out = lay_out(std::min(rows, most), std::min(kMostSplits * rows, most), shape->head_dim, &L);
  return DELTA_OK;
}

int delta_tree_attn(const delta_shape_t* shape, const delta_kv_t* kv, int32_t n_rows, int32_t max_new,
                    const int32_t* row_offsets, const uint32_t* masks, int32_t mask_words, const void* q,
                    void* out, void* ws, size_t ws_bytes, void* stream) {
  ExtendLayout L;
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
  ExtendArgs a = extend_args(shape, kv, L, row_offsets, q, out, ws);
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
  a.n_pieces = std::max(ceil_div(vocab, kMostPiece), std::min({ceil_div(1024, batch), ceil_div(vocab, 2048), kMostPieces}));
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
