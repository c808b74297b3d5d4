// Device-side walk over the runs of a call (see Runs): which sequence a row belongs to.
#pragma once

#include "extend.h"
#include "wave.h"

namespace delta {

__device__ __forceinline__ int run_offset(const Runs& r, int b) {
  return max(0, min(r.row_offsets ? r.row_offsets[b] : b, r.n_rows));
}

// The sequence of a row (wave-uniform), or -1: runs that end at or before the row are counted, one per
// lane (one load for up to 64 sequences, where a binary search would take six dependent ones); of more
// sequences 64 are sampled first.
__device__ __forceinline__ int sequence_of_row(const Runs& r, int row, int lane) {
  if (!r.row_offsets) return row < r.batch ? row : -1;
  int b = 0, size = r.batch;   // the sequence is among b .. b + size - 1, or b + size
  while (size > 64) {
    const int stride = (size + 63) / 64, last = min((lane + 1) * stride, size) - 1;
    const int n = __popcll(__ballot(lane * stride < size && run_offset(r, b + last + 1) <= row));
    b += min(n * stride, size);
    size = min(stride, size - min(n * stride, size));
  }
  b += __popcll(__ballot(lane < size && run_offset(r, b + lane + 1) <= row));
  return b < r.batch && run_offset(r, b) <= row && row < run_offset(r, b + 1) ? b : -1;
}

}  // namespace delta
