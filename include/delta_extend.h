/*
 * delta_extend.h — the prompt side of the paged KV cache of delta_attn.h: runs of new tokens are
 * rotated and appended, and attend to the cache.  C ABI with the conventions of delta_attn.h
 * (memory, errors, layouts, streams): arguments are checked on the host before anything is
 * enqueued, the library never allocates, synchronises or keeps a pointer, and everything it
 * enqueues are kernels, so calls can be captured into HIP graphs.
 *
 * Runs.  A call covers n_rows rows, one per new token, of all sequences one after another: the
 * run of sequence b is rows row_offsets[b] .. row_offsets[b+1]-1 (int32 [batch+1], device memory,
 * the first 0, not decreasing, at most n_rows; a run may be empty).  row_offsets == NULL: one
 * new token per sequence, row b that of sequence b (n_rows == batch).  seq_lens[b] counts the new
 * tokens, so row j of a run of n is token seq_lens[b] - n + j of its sequence.  Rows of no run
 * (behind the last one) are neither read nor written.
 *   Device-side preconditions (not checked): offsets as above; page-table entries of tokens
 *   below seq_lens[b] name pages that exist, and no page that is written belongs to two
 *   sequences.  Offsets are cut to [0, n_rows].
 */
#ifndef DELTA_EXTEND_H
#define DELTA_EXTEND_H

#include "delta_attn.h"

#ifdef __cplusplus
extern "C" {
#endif

/* The position rotation.  Head element pair i of a token at position p turns by the angle
 * p * inv_freq[i]: (x, y) -> (x cos - y sin, y cos + x sin).  The pairs are elements i and
 * i + rotary_dim/2, or with `interleaved` elements 2i and 2i + 1; elements from rotary_dim on
 * stay.  Angles are formed and reduced in fp64, so far positions lose nothing; the rotation is
 * fp32 with one rounding of the result. */
typedef struct {
  const float* inv_freq;      /* fp32 [rotary_dim / 2], device                               */
  const int32_t* positions;   /* int32 [n_rows], device: position of each row's token; NULL:
                                 its index in the sequence                                   */
  int32_t rotary_dim;         /* a multiple of 16, 16 .. head_dim                            */
  int32_t interleaved;        /* 0 or 1                                                      */
} delta_rope_t;

/* Rotates queries and keys of the new tokens, writes keys and values to the paged cache and the
 * rotated queries to q_out (Sec. 2, Eq. gqa_projection and kv_update, for runs of any length).
 *   kv:    the caches are written, in place: row t % 16 of physical page page_table[b, t / 16]
 *          for token t.  bf16 caches hold the values rounded to nearest even; e4m3 caches
 *          value / scale rounded to nearest even, saturated at +-448 (NaN stays NaN).
 *   rope:  NULL: nothing is rotated.
 *   q:     bf16, [n_q_heads, head_dim] per row, q_row_stride ELEMENTS from one row to the next (a
 *          multiple of 8 and at least n_q_heads * head_dim); NULL together with q_out: keys and
 *          values only.  k, v: the same with n_kv_heads.  q, k and v may be views of one
 *          projection's output.
 *   q_out: bf16 [n_rows, n_q_heads, head_dim]; may be q itself where q's rows lie one behind the
 *          other (else DELTA_ERR_INVALID_ARG), and must not overlap the inputs otherwise.
 * q, k, v, q_out and the caches are 16-byte aligned (else DELTA_ERR_INVALID_ARG).  A run whose
 * sequence cannot hold it (seq_lens[b] below the run's length, or above max_pages_per_seq *
 * page_size) is skipped: nothing of it is written.  One kernel launch; no workspace.  n_rows == 0
 * does nothing; 2^24 rows or more, or more than 2^28 query heads in all, give
 * DELTA_ERR_UNSUPPORTED.  Uses all of `shape` but max_seq_len and sm_scale.  A debug build skips
 * tokens whose page-table entry fails its check. */
int delta_rope_append(const delta_shape_t* shape, const delta_kv_t* kv, const delta_rope_t* rope,
                      int32_t n_rows, const int32_t* row_offsets, const void* q,
                      int64_t q_row_stride, const void* k, int64_t k_row_stride, const void* v,
                      int64_t v_row_stride, void* q_out, void* stream);

/* Bytes of workspace that are enough for delta_extend_attn with this shape, for every call of at
 * most n_rows rows and runs of at most max_new (host only): 4 (head_dim + 3) bytes and a little per
 * part of an output, of which a call keeps at most 32 per row and query head and 131072 in all.
 * Calls of more than 65535 tiles give DELTA_ERR_UNSUPPORTED here and in delta_extend_attn: the fewer
 * of batch * ceil(max_new * G / 256) and n_rows * G / 256 + min(batch, n_rows), G query heads per KV
 * head (up to two million rows at G = 8, more at smaller G or in batches of short runs).  So do
 * shapes whose max_seq_len is above 2^31 - 512. */
int delta_extend_workspace_bytes(const delta_shape_t* shape, int32_t n_rows, int32_t max_new,
                                 size_t* out);

/* Causal attention of every new token over its sequence's cached tokens up to itself:
 *   out[row, j, :] = sum_{t <= tau} softmax_t(sm_scale * q[row, j] . k_t) v_t,
 * tau the row's token index; a row whose token index is negative sees no token and gets zeros.
 * The new tokens' keys and values stand in the cache already (delta_rope_append).
 *   q, out:  bf16 [n_rows, n_q_heads, head_dim], 16-byte aligned
 *   max_new: at least the longest run (sizes the grid; with a longer run some rows' outputs are
 *            undefined) and at most n_rows (else DELTA_ERR_INVALID_ARG)
 *   ws:      at least delta_extend_workspace_bytes() bytes, 256-byte aligned, of any content;
 *            it keeps nothing between calls.  Calls that share one must not run concurrently.
 *            (A debug build's status word is its first: zero it before the call to read it.)
 * seq_lens[b] may be 0 (with an empty run) and is cut to max_seq_len.
 * max_seq_len decides the speed of calls of few rows, never their results: a sequence's tokens are
 * cut into pieces for workgroups of their own by this bound, not by seq_lens.  Where it is 4 to 32
 * times the lengths such a call takes up to 2.7 times as long (32/8 heads, one sequence of 4096
 * tokens, 8 new: 16 us with a bound of 4096, 45 with 131072; 512 new behind 7680: 94 with 8192, 240
 * with 32768).  Calls that fill the GPU without pieces, as long prompts do, take the same time.
 * What a row does not see does not reach it, infinite and NaN keys and values of later tokens and of
 * rows past the sequence among it; those that it sees can make its outputs infinite or NaN (a value
 * its own element, a key all), and a NaN query its own outputs.
 * bf16 queries, fp32 scores, softmax and sums, one bf16 rounding of the result; the probabilities
 * are rounded to bf16 before they meet the values (at most 2^-8 of each), their sum is not.  (The
 * decode step's attention of a single token keeps them in three bf16 terms.)  Deterministic: the
 * same call gives the same bits. */
int delta_extend_attn(const delta_shape_t* shape, const delta_kv_t* kv, int32_t n_rows,
                      int32_t max_new, const int32_t* row_offsets, const void* q, void* out,
                      void* ws, size_t ws_bytes, void* stream);

#ifdef __cplusplus
}
#endif

#endif /* DELTA_EXTEND_H */
