// Positions and visible rows of trees of drafted tokens, from the rows' parents.
//
// Work.  A workgroup takes a sequence: its parents go to LDS, then a thread takes a row and goes up to
// the root.  Parents come before their children, so the places that it meets descend, and the mask's
// words are filled and written from the last to the first, one at a time, in a register.
//
// Bound: launch and the chain offsets -> parents -> way up (a step of the way is one LDS read): one tree of 16 rows
// 1.8 us, 96 of 20 to 64 rows 4.1.
#include <algorithm>

#include "drafts.h"
#include "runs.h"

namespace delta {
namespace {

__global__ __launch_bounds__(kMostDrafts) void tree_layout_kernel(const TreeLayoutArgs a) {
  __shared__ int16_t s_parent[kMostDrafts];
  const int b = blockIdx.x, T = blockDim.x;
  const int begin = run_offset(a.runs, b), n_run = run_offset(a.runs, b + 1) - begin;
  const int n = min(n_run, a.max_new);   // (n_run < 0 does nothing)
  for (int j = threadIdx.x; j < n; j += T) {
    const int p = a.parents[begin + j];
    s_parent[j] = (int16_t)(p >= 0 && p < j ? p : -1);
  }
  __syncthreads();
  for (int j = threadIdx.x; j < n; j += T) {
    int depth = 0;
    if (a.masks) {
      uint32_t* mask = a.masks + (size_t)(begin + j) * a.mask_words;
      int word = a.mask_words - 1;
      uint32_t bits = 0;
      for (int i = j;; ++depth) {
        for (; word > i >> 5; --word) {
          mask[word] = bits;
          bits = 0;
        }
        bits |= 1u << (i & 31);
        if ((i = s_parent[i]) < 0) break;
      }
      for (; word >= 0; --word) {
        mask[word] = bits;
        bits = 0;
      }
    } else {
      for (int i = s_parent[j]; i >= 0; i = s_parent[i]) ++depth;
    }
    if (a.positions) a.positions[begin + j] = a.runs.seq_lens[b] - n_run + depth;
  }
}

}  // namespace

hipError_t launch_tree_layout(const TreeLayoutArgs& a, hipStream_t stream) {
  const int threads = std::min(kMostDrafts, (a.max_new + 63) / 64 * 64);
  hipLaunchKernelGGL(tree_layout_kernel, dim3(a.runs.batch), dim3(threads), 0, stream, a);
  return hipGetLastError();
}

}  // namespace delta
