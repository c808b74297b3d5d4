// Argument checks and small helpers shared by the C ABI sources.
#pragma once

#include <math.h>
#include <stdint.h>

#include "../../include/delta_attn.h"
#include "internal.h"

namespace delta {

constexpr size_t kAlign = 256;

inline size_t align_up(size_t x) { return (x + kAlign - 1) / kAlign * kAlign; }
inline int ceil_div(int a, int b) { return (int)(((int64_t)a + b - 1) / b); }

inline int check_shape(const delta_shape_t* s) {
  if (!s) return DELTA_ERR_INVALID_ARG;
  if (s->batch < 1 || s->n_q_heads < 1 || s->n_kv_heads < 1 || s->max_seq_len < 1 ||
      s->max_pages_per_seq < 1 || !(s->sm_scale >= 0.f) || isinf(s->sm_scale))
    return DELTA_ERR_INVALID_ARG;
  if (s->n_q_heads % s->n_kv_heads != 0) return DELTA_ERR_INVALID_ARG;
  if ((int64_t)s->max_seq_len > (int64_t)s->max_pages_per_seq * 16) return DELTA_ERR_INVALID_ARG;
  if (s->page_size != 16) return DELTA_ERR_UNSUPPORTED;
  if (s->head_dim != 64 && s->head_dim != 128) return DELTA_ERR_UNSUPPORTED;
  const int G = s->n_q_heads / s->n_kv_heads;
  if (G > kMaxGroup) return DELTA_ERR_UNSUPPORTED;
  if ((int64_t)s->batch * s->n_q_heads > (1 << 24) || s->batch > 65535 || s->n_kv_heads > 65535)
    return DELTA_ERR_UNSUPPORTED;
  return DELTA_OK;
}

inline int check_kv(const delta_kv_t* kv) {
  if (!kv || !kv->k_cache || !kv->v_cache || !kv->page_table || !kv->seq_lens || kv->n_pages < 0)
    return DELTA_ERR_INVALID_ARG;
  if (kv->kv_type != DELTA_KV_BF16 && kv->kv_type != DELTA_KV_E4M3) return DELTA_ERR_INVALID_ARG;
  // (scales of a bf16 cache would be ignored: refused instead)
  if (kv->kv_type == DELTA_KV_BF16 && (kv->k_scale || kv->v_scale)) return DELTA_ERR_INVALID_ARG;
  // (bytes may start anywhere; the kernels load 16 of them at a time)
  if (kv->kv_type == DELTA_KV_E4M3 &&
      (reinterpret_cast<uintptr_t>(kv->k_cache) | reinterpret_cast<uintptr_t>(kv->v_cache)) % 16)
    return DELTA_ERR_INVALID_ARG;
  return DELTA_OK;
}

inline bool is_e4m3(const delta_kv_t* kv) { return kv->kv_type == DELTA_KV_E4M3; }

inline float scale_log2(const delta_shape_t* s) {
  const float sc = s->sm_scale > 0.f ? s->sm_scale : 1.0f / sqrtf((float)s->head_dim);
  return sc * 1.4426950408889634f;
}

inline int hip_rc(hipError_t e) { return e == hipSuccess ? DELTA_OK : DELTA_ERR_HIP; }

}  // namespace delta
