// Device-side walk over the runs of a call (see Runs): which sequence a row belongs to.
#pragma once

#include "extend.h"
#include "wave.h"

namespace delta {

__device__ __forceinline__ int run_offset(const Runs& r, int b) {
  return max(0, min(r.row_offsets ? r.row_offsets[b] : b, r.n_rows));
}

// The sequence of a row (wave-uniform), or -1: sequences whose run ends at or before the row are
// counted, 64 at a time, one per lane (one load for up to 64 sequences; a binary search would take
// six dependent ones).
__device__ __forceinline__ int sequence_of_row(const Runs& r, int row, int lane) {
  if (!r.row_offsets) return row < r.batch ? row : -1;
  int b = 0;
  for (int c = 0; c < r.batch; c += 64) {
    const bool ended = c + lane < r.batch && run_offset(r, c + lane + 1) <= row;
    const int n = __popcll(__ballot(ended));
    b += n;
    if (n < 64) break;
  }
  return b < r.batch && run_offset(r, b) <= row ? b : -1;
}

}  // namespace delta
