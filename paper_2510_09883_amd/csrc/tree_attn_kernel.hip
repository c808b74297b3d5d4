// Attention of trees of drafted tokens over the paged cache: every row of a run sees the tokens before
// the run and the rows of the run that its mask names.
//
// The mathematics, the tile step and the LDS layouts are attend_runs.h's; a row's mask is looked at only in
// the blocks that hold rows of the run.
#include "attend_runs.h"
#include "drafts.h"

namespace delta {
namespace {

// Tiles of 32 rows, four waves along the keys.
template <int D, bool KV8>
__global__ __launch_bounds__(256, 2) void tree_few_kernel(const ExtendArgs a) {
  __shared__ __attribute__((aligned(256))) uint16_t s_kv[kBodyLds<D, 1, 4, 1> / 2];
  __shared__ float2 s_ml[4 * 64];
  TileOf t;
  if (find_tile<32>(a, t)) extend_body<D, 1, 4, 1, KV8, true>(a, t, s_kv, s_ml, nullptr);
}

// Tiles of 256 rows, eight waves along them.
template <int D, bool KV8>
__global__ __launch_bounds__(512, 1) void tree_many_kernel(const ExtendArgs a) {
  __shared__ __attribute__((aligned(256))) uint16_t s_kv[kBodyLds<D, 8, 1, 2> / 2];
  __shared__ int s_others;   // some wave has met infinite or NaN values in an edge block
  TileOf t;
  if (!find_tile<256>(a, t)) return;
  if (threadIdx.x == 0) s_others = 0;   // (the walk's first barrier is before any use)
  extend_body<D, 8, 1, 2, KV8, true>(a, t, s_kv, nullptr, &s_others);
}

template <int D, bool KV8>
hipError_t launch_d(const ExtendPlan& p, const ExtendArgs& a, hipStream_t stream) {
  const dim3 grid(a.n_kv_heads, p.tiles, p.n_split);
  if (p.rows == 32) hipLaunchKernelGGL((tree_few_kernel<D, KV8>), grid, dim3(256), 0, stream, a);
  else hipLaunchKernelGGL((tree_many_kernel<D, KV8>), grid, dim3(512), 0, stream, a);
  hipError_t e = hipGetLastError();
  if (e != hipSuccess || p.n_split == 1) return e;
  const int64_t items = (int64_t)a.runs.n_rows * a.n_q_heads;
  const int per = 256 / (D / 4);
  hipLaunchKernelGGL(extend_join_kernel<D>, dim3((unsigned)((items + per - 1) / per)), dim3(256), 0, stream, a, KV8);
  return hipGetLastError();
}

}  // namespace

hipError_t launch_tree_attn(const ExtendPlan& p, int head_dim, bool kv8, const ExtendArgs& a, hipStream_t stream) {
  if (head_dim == 128) return kv8 ? launch_d<128, true>(p, a, stream) : launch_d<128, false>(p, a, stream);
  return kv8 ? launch_d<64, true>(p, a, stream) : launch_d<64, false>(p, a, stream);
}

}  // namespace delta
