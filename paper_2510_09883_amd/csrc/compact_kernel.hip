// Keeping the accepted rows of drafted runs: key and value rows move together in the caches of all layers.
//
// Work.  A workgroup takes a sequence in a layer.  A path ascends, so path[i] >= i, and where path[i] = i
// nothing moves: that is a beginning of the path.  The places of the rest go to LDS, as byte offsets into
// a cache; then a thread takes 16 bytes of a head's row, of K or V, and moves them for all rows of the path in
// its order: a row is written by the thread that has read it, or read a row behind it, before (path[i + 1] >
// path[i] >= i), and eight rows are in flight at once for the same reason.
//
// Bound: launch and the chain offsets and path -> pages -> rows -> stores: one sequence in 28 layers 4.7 us, 64 in
// 28 layers, 190 KB a layer to move, 6.4 us.
#include "debug_check.h"
#include "drafts.h"
#include "runs.h"

namespace delta {
namespace {

constexpr int kThreads = 256;
constexpr int kInFlight = 8;

typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));

struct Kept {
  bool ok;      // the sequence is compacted (else it is left alone)
  int before;   // tokens before the run
  int n;        // rows kept
  int first;    // the first of them that moves
};

// What a workgroup (all threads call it) keeps of sequence b's run.
__device__ __forceinline__ Kept kept_of(const CompactArgs& a, int b) {
  const int begin = run_offset(a.runs, b), run = run_offset(a.runs, b + 1) - begin;
  const int s = a.runs.seq_lens[b], n = a.n_path[b];
  const int32_t* path = a.path + (size_t)b * a.max_new;
  Kept k{run >= 0 && s >= run && s <= (int64_t)16 * a.runs.max_pages && n >= 0 && n <= min(run, a.max_new), s - run, n, 0};
  int same = 0;
  bool fits = true;
  if (k.ok) {   // (the same for all threads)
    for (int i = threadIdx.x; i < n; i += kThreads) {
      const int p = path[i];
      fits &= p >= 0 && p < run && (i == 0 || p > path[i - 1]);
      same += p == i;
    }
  }
  k.ok &= __syncthreads_and(fits) != 0;
  __shared__ int s_first;
  if (threadIdx.x == 0) s_first = 0;
  __syncthreads();
  if (same) atomicAdd(&s_first, same);
  __syncthreads();
  k.first = s_first;
  return k;
}

__global__ __launch_bounds__(kThreads) void compact_kernel(const CompactArgs a) {
  __shared__ int64_t s_from[kMostDrafts], s_to[kMostDrafts];   // element offsets of head 0's rows; -1: none
  const int b = blockIdx.y, layer = blockIdx.x;
  const Kept k = kept_of(a, b);
  if (a.new_lens && layer == 0 && threadIdx.x == 0) a.new_lens[b] = k.ok ? k.before + k.n : a.runs.seq_lens[b];
  if (!k.ok || k.first >= k.n) return;
  const CompactLayer& L = a.layers[layer];
  const int32_t* table = L.page_table + (size_t)b * a.runs.max_pages;
  const int32_t* path = a.path + (size_t)b * a.max_new;
  const int64_t page_stride = (int64_t)a.n_kv_heads * 16 * a.head_dim;
  for (int i = k.first + threadIdx.x; i < k.n; i += kThreads) {
    const int from = k.before + path[i], to = k.before + i;
    const int p0 = table[from >> 4], p1 = table[to >> 4];
    const bool bad = DELTA_DEBUG && (p0 < 0 || p1 < 0 || (L.n_pages > 0 && (p0 >= L.n_pages || p1 >= L.n_pages)));
    s_from[i] = bad ? -1 : (int64_t)p0 * page_stride + (from & 15) * a.head_dim;
    s_to[i] = (int64_t)p1 * page_stride + (to & 15) * a.head_dim;
  }
  __syncthreads();
  const int bytes = a.e4m3 >> layer & 1 ? 1 : 2;
  const int per_row = a.head_dim * bytes / 16;       // 16-byte pieces of a head's row
  const int pieces = a.n_kv_heads * per_row;         // of a token in K (or V)
  for (int u = threadIdx.x; u < 2 * pieces; u += kThreads) {
    const bool is_v = u >= pieces;
    const int c = is_v ? u - pieces : u, h = c / per_row, e = c - h * per_row;
    uint8_t* at = (is_v ? L.v_cache : L.k_cache) + (size_t)h * 16 * a.head_dim * bytes + 16 * e;
    for (int i0 = k.first; i0 < k.n; i0 += kInFlight) {
      u32x4 x[kInFlight];
#pragma unroll
      for (int i = 0; i < kInFlight; ++i)
        if (i0 + i < k.n && s_from[i0 + i] >= 0) x[i] = *reinterpret_cast<const u32x4*>(at + s_from[i0 + i] * bytes);
#pragma unroll
      for (int i = 0; i < kInFlight; ++i)
        if (i0 + i < k.n && s_from[i0 + i] >= 0) *reinterpret_cast<u32x4*>(at + s_to[i0 + i] * bytes) = x[i];
    }
  }
}

// The new lengths alone, where they take the old ones' place: after all that read those.
__global__ __launch_bounds__(kThreads) void compact_lens_kernel(const CompactArgs a) {
  const int b = blockIdx.x;
  const Kept k = kept_of(a, b);
  if (k.ok && threadIdx.x == 0) a.new_lens[b] = k.before + k.n;
}

}  // namespace

hipError_t launch_compact(const CompactArgs& a, hipStream_t stream) {
  hipLaunchKernelGGL(compact_kernel, dim3(a.n_layers, a.runs.batch), dim3(kThreads), 0, stream, a);
  return hipGetLastError();
}

hipError_t launch_compact_lens(const CompactArgs& a, hipStream_t stream) {
  hipLaunchKernelGGL(compact_lens_kernel, dim3(a.runs.batch), dim3(kThreads), 0, stream, a);
  return hipGetLastError();
}

}  // namespace delta
