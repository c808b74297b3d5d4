/*
 * delta_drafts.h — a round of drafted tokens over the paged KV cache of delta_attn.h.  The drafts of a
 * sequence form a tree: several continuations of one token may be tried at once.  In the order of use:
 * delta_tree_layout (once a round), in every layer delta_norm_rope_append (or delta_rope_append) and
 * delta_tree_attn, then delta_verify_drafts and delta_cache_compact.  C ABI with the conventions of
 * delta_attn.h (memory, errors, layouts, streams) and the runs of delta_extend.h: arguments are checked on
 * the host before anything is enqueued, the library never allocates, synchronises or keeps a pointer, and
 * everything it enqueues are kernels, so calls can be captured into HIP graphs.
 *
 * Trees.  The rows of a run are the nodes of its tree, a parent before its children: parents[row] (int32,
 * device memory) is the place in the run (0 for its first row) of the row that this one continues, or -1: it
 * continues the cached tokens before the run.  An entry outside [0, place of the row) counts as -1.  Where
 * drafts are verified, a run's first row is the token that was decided last and whose key and value are not
 * cached yet, and the others are drafts that continue it.  The token of place j stands in the cache at index
 * P + j, P = seq_lens[b] - n tokens before a run of n.
 */
#ifndef DELTA_DRAFTS_H
#define DELTA_DRAFTS_H

#include "delta_attn.h"
#include "delta_extend.h"

#ifdef __cplusplus
extern "C" {
#endif

/* The longest run of a tree: larger max_new give DELTA_ERR_UNSUPPORTED. */
#define DELTA_MOST_DRAFTS 512

/* Norms of the heads of queries and keys: x becomes w * x / sqrt(mean(x^2) + eps) over a head's elements,
 * in fp32 (elements past 2^60 overflow its squares). */
enum { DELTA_NORM_BF16 = 0, DELTA_NORM_F32 = 1 };
typedef struct {
  const void* q_weight;       /* [head_dim] of weight_type, device, 16-byte aligned; NULL: 1 */
  const void* k_weight;       /* the same                                                    */
  int32_t weight_type;        /* DELTA_NORM_BF16 or DELTA_NORM_F32                           */
  float eps;                  /* finite, >= 0                                                */
} delta_norm_t;

/* delta_rope_append with the heads of q and k normed before they turn, in the same pass: norm and rotation
 * are fp32 with one rounding of the result.  norm: not NULL.  All else as delta_rope_append; with a tree,
 * rope->positions are those of delta_tree_layout, as a row's depth and not its place decides its angle. */
int delta_norm_rope_append(const delta_shape_t* shape, const delta_kv_t* kv, const delta_norm_t* norm,
                           const delta_rope_t* rope, int32_t n_rows, const int32_t* row_offsets, const void* q,
                           int64_t q_row_stride, const void* k, int64_t k_row_stride, const void* v,
                           int64_t v_row_stride, void* q_out, void* stream);

/* What follows from the parents, for all layers of a round:
 *   positions: int32 [n_rows]: P + the row's depth (0 for a parent of -1); NULL: not written
 *   masks:     uint32 [n_rows, mask_words]: bit i of a row (bit i % 32 of word i / 32) is set for the
 *              places i of the row itself and of the rows that it continues; NULL: not written
 *   seq_lens:  int32 [batch], counting the run; read for positions only (else NULL)
 *   max_new:   at least the longest run, at most 32 * mask_words (with masks) and n_rows; places from
 *              max_new on are not written.
 * One kernel launch, no workspace.  Uses batch of `shape`. */
int delta_tree_layout(const delta_shape_t* shape, const int32_t* seq_lens, int32_t n_rows, int32_t max_new,
                      const int32_t* row_offsets, const int32_t* parents, int32_t* positions, uint32_t* masks,
                      int32_t mask_words, void* stream);

/* Bytes of workspace that are enough for delta_tree_attn with this shape, for every call of at most n_rows
 * rows and runs of at most max_new (host only). */
int delta_tree_workspace_bytes(const delta_shape_t* shape, int32_t n_rows, int32_t max_new, size_t* out);

/* Attention of every row of a run to the P cached tokens before the run and to the rows of the run whose
 * bits its mask has:
 *   out[row, j, :] = sum_{t in seen(row)} softmax_t(sm_scale * q[row, j] . k_t) v_t;
 * a row that sees no token gets zeros.
 *   masks:      uint32 [n_rows, mask_words], as delta_tree_layout writes them or any other; bits of places
 *               from the run's length on are ignored.  A row sees itself only if its own bit is set.
 *   mask_words: >= 1 and at least max_new / 32, rounded up
 *   q, out, max_new, ws, and what is undefined with a run longer than max_new: as in delta_extend_attn, so
 *   also infinite and NaN keys and values (a row gets them of the tokens that it sees, and no others) and
 *   determinism.  Calls of more than 65535 tiles (as counted there) give DELTA_ERR_UNSUPPORTED.
 * Up to 256 sequences are shared out over the GPU by their lengths; of more, a workgroup walks a sequence alone,
 * and the longest decides (8 rows each, 32/8 heads, one of 65536 tokens among 300s: 160 us for 256 sequences, 708
 * for 257; where all are 500 to 8192 tokens long 805 and 791).  max_seq_len decides how a call is cut: far above the
 * lengths it takes up to 1.7 times as long (16 sequences of 300 to 700 tokens, 16 rows, 32/8 heads: 17 us with 700, 29
 * with 1400 and more; one of 2048, 64 rows: 21 and 25; one of 8192, 16 rows: 21 and 23), and calls that fill the GPU
 * the same time.
 * bf16 queries, fp32 scores, softmax and sums, one bf16 rounding of the result.  Where they meet the values
 * (their sum is not rounded) the probabilities have 16 bits: over e4m3 caches those of fp16 (at most 2^-11 of
 * each); over bf16 caches two bf16 terms (2^-16) where runs have up to 32 rows a KV head (max_new * G, G query
 * heads per KV head) or the batch has little to walk, else one (2^-8). */
int delta_tree_attn(const delta_shape_t* shape, const delta_kv_t* kv, int32_t n_rows, int32_t max_new,
                    const int32_t* row_offsets, const uint32_t* masks, int32_t mask_words, const void* q,
                    void* out, void* ws, size_t ws_bytes, void* stream);

/* Bytes of workspace that are enough for delta_verify_drafts with this many sequences or fewer and this
 * vocabulary or a smaller one (host only). */
int delta_verify_workspace_bytes(int32_t batch, int32_t vocab, size_t* out);

/* Which drafts the target's probabilities accept, and the token after them, so that what is kept is
 * distributed as the target's own samples are.  From the run's first row on, the rows that continue the
 * current row are tried in ascending order.  Let p be the target's probabilities after the current row, q the
 * drafting model's, from which the drafts were drawn, x a draft's token and u its uniform number; r = p and
 * R = 1 at first.  The draft is accepted, and becomes the current row, where
 *     u * q(x) * R < r(x);
 * otherwise r becomes max(r - R q, 0) and R its sum, and the next one is tried.  draft == NULL: the drafts
 * were not drawn but chosen; q counts as 1 at the draft's own token and 0 elsewhere, so that after a
 * rejection r(x) = 0 and R is less by what it was (never less than 0).  After the last accepted row comes the
 * token
 *     next = the smallest v with r(0) + .. + r(v) > u0 * (r(0) + .. + r(vocab - 1)),
 * u0 the uniform number of the run's first row (the last token with r > 0 if there is no such v).  Where r is
 * 0 everywhere, p takes its place; where p is too, next is -1.  Negative and NaN probabilities count as 0.
 * A sum R over a whole row is formed only where a drawn sibling is tried after a rejection, and then by every
 * workgroup of the sequence (13 us for 151936 tokens).
 * Formed in fp64 from fp32 inputs, so a choice depends on the order of sums only where u0 times the sum meets
 * a partial sum to about 1e-15.
 *   target:  fp32 [n_rows, vocab]: probabilities after each row, target_row_stride ELEMENTS from one row to
 *            the next (>= vocab); each row sums to 1 (for the test of a draft; next divides by the sum)
 *   draft:   the same, of the drafting model; rows that no other row continues are not read.  NULL: none.
 *   tokens:  int32 [n_rows]; a run's first is not read.  One outside [0, vocab) has probability 0.
 *   parents: int32 [n_rows], as above; a row other than the first with a parent of -1 is never tried
 *   uniform: fp32 [n_rows] in [0, 1)
 *   path:    int32 [batch, max_new]: the places of the accepted rows in their runs, ascending, the first
 *            row's (0) among them; -1 from the count on
 *   n_path:  int32 [batch]: their count (0: the run is empty, next is -1)
 *   next:    int32 [batch]
 *   max_new: at least the longest run, at least 1 and at most n_rows (of longer runs the rest is not tried)
 *   ws:      256-byte aligned, of any content; it keeps nothing between calls.  Calls that share one must not
 *            run concurrently.
 * Two kernel launches.  batch at most 65535, vocab at most 2^20 and n_rows below 2^24, else DELTA_ERR_UNSUPPORTED. */
int delta_verify_drafts(int32_t batch, int32_t n_rows, int32_t max_new, const int32_t* row_offsets, int32_t vocab,
                        const float* target, int64_t target_row_stride, const float* draft,
                        int64_t draft_row_stride, const int32_t* tokens, const int32_t* parents,
                        const float* uniform, int32_t* path, int32_t* n_path, int32_t* next, void* ws,
                        size_t ws_bytes, void* stream);

/* Keeps the accepted rows of every run and drops the others, in the caches of all layers: the key and value
 * rows of token P + path[b, i] move to token P + i, i < n_path[b], in every KV head, bit for bit.
 *   kv:       HOST array of n_layers descriptors; the caches are written in place.  kv_type may differ from
 *             layer to layer, and page_table too; seq_lens is one for all (else DELTA_ERR_INVALID_ARG) and
 *             counts the runs.  All caches are different ones (else DELTA_ERR_INVALID_ARG).
 *   path, n_path: as delta_verify_drafts writes them: path int32 [batch, max_new]
 *   max_new:  at least 1 and at most n_rows
 *   new_lens: int32 [batch]: P + n_path[b]; may be the layers' seq_lens; NULL: not written.
 * A sequence is left alone, and its new length is its old one, where the path is not ascending places of its
 * run, or the count is not in [0, min(run, max_new)], or the sequence cannot hold the run (seq_lens[b] below
 * its length or above max_pages_per_seq * page_size).  No page that is written may belong to two sequences.
 * One kernel launch for up to 64 layers, and one more where new_lens is seq_lens; no workspace.  Caches are
 * 16-byte aligned (else DELTA_ERR_INVALID_ARG).  Uses all of `shape` but max_seq_len, n_q_heads and sm_scale.
 * A debug build leaves out moves whose page-table entries fail its check. */
int delta_cache_compact(const delta_shape_t* shape, int32_t n_layers, const delta_kv_t* kv, int32_t n_rows,
                        int32_t max_new, const int32_t* row_offsets, const int32_t* path, const int32_t* n_path,
                        int32_t* new_lens, void* stream);

#ifdef __cplusplus
}
#endif

#endif /* DELTA_DRAFTS_H */
