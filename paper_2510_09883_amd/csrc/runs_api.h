// Argument checks of the C ABI calls over runs of rows.
#pragma once

#include <algorithm>

#include "api_common.h"
#include "extend.h"

namespace delta {

inline bool aligned(const void* p, uintptr_t to) { return reinterpret_cast<uintptr_t>(p) % to == 0; }

inline int check_runs(const delta_shape_t* s, int32_t n_rows, const int32_t* row_offsets) {
  if (n_rows < 0) return DELTA_ERR_INVALID_ARG;
  if (!row_offsets && n_rows != s->batch) return DELTA_ERR_INVALID_ARG;
  if ((int64_t)n_rows * s->n_q_heads > (1 << 28)) return DELTA_ERR_UNSUPPORTED;
  return DELTA_OK;
}

inline Runs runs_of(const delta_shape_t* s, const delta_kv_t* kv, int32_t n_rows, const int32_t* row_offsets) {
  return Runs{row_offsets, kv->seq_lens, kv->page_table, n_rows, s->batch, s->max_pages_per_seq};
}

// Most tiles of a call: a launch's second grid size.
constexpr int kMostTiles = 65535;
// The longest bound of a sequence: the kernels round key indices up to whole blocks, of 256 keys at
// most, in 32 bits.
constexpr int kMostKeys = INT32_MAX - 511;

// The kernels' arguments of an attention call whose own have been checked, but for the cut and the workspace.
inline ExtendArgs extend_args(const delta_shape_t* shape, const delta_kv_t* kv, int n_rows, const int32_t* row_offsets,
                              const void* q, void* out) {
  ExtendArgs a{};
  a.runs = runs_of(shape, kv, n_rows, row_offsets);
  a.k_cache = static_cast<const uint8_t*>(kv->k_cache);
  a.v_cache = static_cast<const uint8_t*>(kv->v_cache);
  a.k_scale = kv->k_scale;
  a.v_scale = kv->v_scale;
  a.q = static_cast<const uint16_t*>(q);
  a.out = static_cast<uint16_t*>(out);
  a.page_stride = (int64_t)shape->n_kv_heads * 16 * shape->head_dim;
  a.n_q_heads = shape->n_q_heads;
  a.n_kv_heads = shape->n_kv_heads;
  a.max_seq_len = shape->max_seq_len;
  a.n_split = 1;
  a.scale_log2 = scale_log2(shape);
  a.n_pages = kv->n_pages;
  return a;
}

// Checks the arguments of delta_rope_append and fills *a (not with n_rows == 0, which does nothing).
inline int append_args(const delta_shape_t* shape, const delta_kv_t* kv, const delta_rope_t* rope, int32_t n_rows,
                       const int32_t* row_offsets, const void* q, int64_t q_row_stride, const void* k,
                       int64_t k_row_stride, const void* v, int64_t v_row_stride, void* q_out, RopeAppendArgs* a) {
  int rc = check_shape(shape);
  if (rc) return rc;
  if ((rc = check_kv(kv))) return rc;
  if ((rc = check_runs(shape, n_rows, row_offsets))) return rc;
  if (n_rows >= 1 << 24) return DELTA_ERR_UNSUPPORTED;   // (a launch has fewer than 2^32 threads)
  if (rope) {
    if (!rope->inv_freq || rope->rotary_dim < 16 || rope->rotary_dim > shape->head_dim ||
        rope->rotary_dim % 16 || (rope->interleaved != 0 && rope->interleaved != 1))
      return DELTA_ERR_INVALID_ARG;
  }
  if (n_rows == 0) return DELTA_OK;
  if (!k || !v || !q != !q_out) return DELTA_ERR_INVALID_ARG;
  const int64_t q_row = (int64_t)shape->n_q_heads * shape->head_dim;
  const int64_t kv_row = (int64_t)shape->n_kv_heads * shape->head_dim;
  if (k_row_stride < kv_row || k_row_stride % 8 || v_row_stride < kv_row || v_row_stride % 8 ||
      (q && (q_row_stride < q_row || q_row_stride % 8)))
    return DELTA_ERR_INVALID_ARG;
  // (in place, rows that stand apart would be written over rows still to be read)
  if (q && q == q_out && q_row_stride != q_row && n_rows > 1) return DELTA_ERR_INVALID_ARG;
  for (const void* p : {q, k, v, static_cast<const void*>(q_out), kv->k_cache, kv->v_cache})
    if (!aligned(p, 16)) return DELTA_ERR_INVALID_ARG;
  a->runs = runs_of(shape, kv, n_rows, row_offsets);
  // (the cache descriptor is shared with the calls that only read it)
  a->k_cache = static_cast<uint8_t*>(const_cast<void*>(kv->k_cache));
  a->v_cache = static_cast<uint8_t*>(const_cast<void*>(kv->v_cache));
  a->k_scale = kv->k_scale;
  a->v_scale = kv->v_scale;
  a->q = static_cast<const uint16_t*>(q);
  a->k = static_cast<const uint16_t*>(k);
  a->v = static_cast<const uint16_t*>(v);
  a->q_out = static_cast<uint16_t*>(q_out);
  a->q_stride = q_row_stride;
  a->k_stride = k_row_stride;
  a->v_stride = v_row_stride;
  a->page_stride = (int64_t)shape->n_kv_heads * 16 * shape->head_dim;
  if (rope) {
    a->inv_freq = rope->inv_freq;
    a->positions = rope->positions;
    a->rotary_dim = rope->rotary_dim;
    a->interleaved = rope->interleaved;
  }
  a->n_q_heads = q ? shape->n_q_heads : 0;
  a->n_kv_heads = shape->n_kv_heads;
  a->n_pages = kv->n_pages;
  return DELTA_OK;
}

}  // namespace delta
