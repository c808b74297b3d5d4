// Internal interface between drafts_api.cpp and the kernels for a round of drafted tokens
// (tree_layout_kernel.hip, tree_attn_kernel.hip, verify_kernel.hip, compact_kernel.hip).
#pragma once

#include "../../include/delta_drafts.h"
#include "extend.h"

namespace delta {

constexpr int kMostDrafts = DELTA_MOST_DRAFTS;

struct TreeLayoutArgs {
  Runs runs;                 // (page_table unused; seq_lens may be null without positions)
  const int32_t* parents;    // [n_rows]
  int32_t* positions;        // [n_rows] or null
  uint32_t* masks;           // [n_rows, mask_words] or null
  int32_t mask_words, max_new;
};

hipError_t launch_tree_layout(const TreeLayoutArgs& a, hipStream_t stream);

// How an attention call over trees is cut: tiles of `rows` (token, query head of the group) rows per (sequence,
// KV head).  Up to kCutBatch sequences: groups of n_kv_heads workgroups share the work evenly, from the sequences'
// lengths; more sequences: a workgroup per tile and KV head.
constexpr int kCutBatch = 256;
// Work is counted in units of about 0.14 us: a tile costs kTileUnits and more for each block of its keys
// (tree_attn_kernel.hip), and a group takes at least kLeastUnits.
constexpr int kTileUnits = 40, kLeastUnits = 16, kMostUnits64 = 6;   // (kMostUnits64: of 64 keys)
struct TreePlan {
  int rows = 0;         // 32 or 256
  int tiles = 0;        // most tiles of a call
  int workgroups = 0;   // groups * n_kv_heads, at most 1023 groups; 0: not shared
  bool pieces = false;  // a group takes a piece of one tile, else an equal part of all
};

TreePlan plan_tree(const delta_shape_t* s, int n_rows, int max_new);
hipError_t launch_tree_attn(const TreePlan& p, int head_dim, bool kv8, const ExtendArgs& a, hipStream_t stream);

// Pieces of a row of probabilities, each taken by a workgroup of eight waves, and the elements of a piece and of a
// wave's part of it.
constexpr int kMostPieces = 64, kVerifyWaves = 8, kMostPart = 2048, kMostPiece = kVerifyWaves * kMostPart;
constexpr int kMostVocab = kMostPieces * kMostPiece;

// A sequence's part of the workspace, from the first launch to the second.
struct VerifyState {
  int32_t cur, k;                            // the last accepted row and the rejections at it
  double S;                                  // the sum of R before each of them, of drawn drafts
  double sums[kMostPieces * kVerifyWaves];   // a part's sum of r
};

struct VerifyArgs {
  Runs runs;                 // (only the offsets; n_rows, batch)
  const float* target;       // rows target_stride elements apart
  const float* draft;        // or null
  int64_t target_stride, draft_stride;
  const int32_t* tokens;     // [n_rows]
  const int32_t* parents;
  const float* uniform;
  int32_t* path;             // [batch, max_new]
  int32_t* n_path;           // [batch]
  int32_t* next;             // [batch]
  VerifyState* state;        // [batch]
  int32_t vocab, max_new;
  int32_t part;              // elements of a wave's part: a multiple of for_row's round
  int32_t n_pieces;          // workgroups per sequence
};

hipError_t launch_verify(const VerifyArgs& a, hipStream_t stream);

// Layers of one launch of the compaction (their pointers are kernel arguments).
constexpr int kLayersPerLaunch = 64;

struct CompactLayer {
  uint8_t* k_cache;          // [pages, Hkv, 16, D], 1 or 2 bytes an element
  uint8_t* v_cache;
  const int32_t* page_table; // [B, max_pages]
  int64_t n_pages;           // 0: not stated; debug checks
};

struct CompactArgs {
  Runs runs;                 // (page_table unused)
  const int32_t* path;       // [batch, max_new]
  const int32_t* n_path;     // [batch]
  int32_t* new_lens;         // [batch] or null
  int32_t max_new, n_kv_heads, head_dim, n_layers;
  uint64_t e4m3;             // bit i: layer i's caches have 1 byte an element
  CompactLayer layers[kLayersPerLaunch];
};

hipError_t launch_compact(const CompactArgs& a, hipStream_t stream);
hipError_t launch_compact_lens(const CompactArgs& a, hipStream_t stream);

}  // namespace delta
