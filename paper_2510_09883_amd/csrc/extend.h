// Internal interface between extend_api.cpp and the kernels for runs of new tokens
// (rope_append_kernel.hip, extend_kernel.hip).
#pragma once

#include "../../include/delta_extend.h"
#include "internal.h"

namespace delta {

// The runs of a call: rows row_offsets[b] .. row_offsets[b + 1] - 1 are sequence b's (null: row b).
struct Runs {
  const int32_t* row_offsets;
  const int32_t* seq_lens;   // [B], counting the new tokens
  const int32_t* page_table; // [B, max_pages]
  int32_t n_rows, batch, max_pages;
};

struct RopeAppendArgs {
  Runs runs;
  uint8_t* k_cache;          // [pages, Hkv, 16, D] of bf16 or e4m3
  uint8_t* v_cache;
  const float* k_scale;      // [Hkv] of an e4m3 cache, or null (1)
  const float* v_scale;
  const uint16_t* q;         // bf16, rows q_stride elements apart; null: no queries
  const uint16_t* k;
  const uint16_t* v;
  uint16_t* q_out;           // bf16 [n_rows, Hq, D]
  int64_t q_stride, k_stride, v_stride;
  int64_t page_stride;       // elements per physical page = Hkv * 16 * D
  const float* inv_freq;     // [rotary_dim / 2]
  const int32_t* positions;  // [n_rows] or null
  int32_t rotary_dim;        // 0: nothing is rotated
  int32_t interleaved;
  int32_t n_q_heads, n_kv_heads;   // (n_q_heads = 0 without queries)
  int64_t n_pages;           // physical pages of the caches (0: not stated); debug checks
};

hipError_t launch_rope_append(int head_dim, bool kv8, const RopeAppendArgs& a, hipStream_t stream);

struct ExtendArgs {
  Runs runs;
  const uint8_t* k_cache;
  const uint8_t* v_cache;
  const float* k_scale;
  const float* v_scale;
  const uint16_t* q;         // bf16 [n_rows, Hq, D]
  uint16_t* out;
  float* part_o;             // [n_split, n_rows, Hq, D] un-normalised outputs of a split
  float* part_ml;            // [n_split, n_rows, Hq, 2] its (max, sum), log2 domain
  int32_t* part_n;           // [n_rows, Hq] pieces of a row's keys; 0: one, whose output is written
  int64_t page_stride;
  int32_t n_q_heads, n_kv_heads;
  int32_t max_seq_len;       // host bound of seq_lens[b] (longer ones are cut to it)
  int32_t n_split;
  int32_t split_keys;        // keys of a piece, a multiple of every kernel's block
  float scale_log2;
  int64_t n_pages;
  uint32_t* status;          // debug status word
};

// How a call is cut: tiles of `rows` (token, query head of the group) rows per (sequence, KV
// head), at most `tiles` of them, each over n_split pieces of the cache.
struct ExtendPlan {
  int rows = 0;
  int tiles = 0;
  int n_split = 1;
  int split_keys = 0;
};

ExtendPlan plan_extend(const delta_shape_t* s, int n_rows, int max_new);
hipError_t launch_extend(const ExtendPlan& p, int head_dim, bool kv8, const ExtendArgs& a, hipStream_t stream);

}  // namespace delta
