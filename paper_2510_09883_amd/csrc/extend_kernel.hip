// Causal attention of runs of new tokens over the paged cache (Sec. 2, Eq. gqa_attention, for more
// than one query token of a sequence).
//
// The mathematics, the tile step and the LDS layouts are attend_runs.h's.
//
// Work.  Two kernels (extend_api.cpp decides which, and the pieces of the keys):
//
//   * many rows: tiles of 256, eight waves along the rows (WR = 8).  All waves bring a block of 64
//     keys to LDS, 16 bytes a thread and load; the next block's loads are in flight, in registers,
//     while one is worked on; two buffers, one barrier a block.  A tile of at most 32 rows (a single
//     token beside prompts) is taken as below, by all eight waves along its keys.
//   * few rows: tiles of 32, four waves along the keys (WK = 4).  Waves share nothing, so each brings
//     its own 32 keys to its own LDS, without barriers, loads the bytes past the caches, and two
//     workgroups fit a CU.  In the end the waves are joined through LDS, each taking a share of the
//     outputs.
//
// Precision.  Scores, maximum, sum and outputs are fp32; a probability is rounded to bf16 for the
// P V product, whose inputs the matrix cores take in 16 bits: at most 2^-8 of each, which in the
// output adds to the result's own rounding (1.7e-3 rms together instead of 1.6e-3, 1.8e-3 where rows see
// a few tokens only).  A second bf16 term per probability, what the first leaves, needs half as many
// products again, of which the many-row kernel has 356 us in the prompt below.  Runs of at most 32 rows,
// which wait for memory, pay for it too, us without and with it, 32/8 heads: 16 sequences of 16384
// tokens, 8 new ones 170 and 172 (e4m3 110 and 124), 8 of 4096, 4 new ones 27.8 and 29.9, 16 of 300, 8
// new ones 9.8 and 10.7.
//
// Bound.  Many rows: the card's power, then the issue of two waves a SIMD.  A prompt of 8192 tokens,
// 32/8 heads: 580-640 us from card to card (860-950 TFLOP/s, where the library's product of 8192 x 8192
// random matrices runs at 1450); 503 with every value zero, at which that product runs at 2100.  The
// products alone take 356 us; reading K and V from LDS 130 of the rest, exponents and maxima 140, moving
// blocks to LDS 90, the barrier 30.  Measured slower or equal: scores of the next 32 keys formed during
// the softmax of these (636), blocks passed by counters instead of a barrier (654), 128-row tiles with
// two workgroups a CU (645), 64 rows a wave, which halves the LDS reads but moves the queries through
// accumulation registers (820), raised priority around the products (635).
// Few rows: HBM, 16 sequences of 4K-16K tokens with up to 8 drafted ones, 32/8 heads, 709 MB: 119 us (6.0
// TB/s) and 4.6 for the join; with ordinary loads 148.
#include "attend_runs.h"

namespace delta {
namespace {

// Tiles of 32 rows, four waves along the keys.
template <int D, bool KV8>
__global__ __launch_bounds__(256, 2) void extend_few_kernel(const ExtendArgs a) {
  __shared__ __attribute__((aligned(256))) uint16_t s_kv[kBodyLds<D, 1, 4, 1> / 2];
  __shared__ float2 s_ml[4 * 64];
  TileOf t;
  Piece p;
  if (find_tile<32>(a, t) && causal_piece<32, 128>(a, t, p))
    extend_body<D, 1, 4, 1, KV8, false>(a, t, p, s_kv, s_ml, nullptr);
}

// Tiles of 256 rows, eight waves along them; a tile that has no more than 32 (a single token beside
// prompts) is taken by eight waves along its keys instead of by one.
template <int D, bool KV8>
__global__ __launch_bounds__(512, 1) void extend_many_kernel(const ExtendArgs a) {
  __shared__ __attribute__((aligned(256))) uint16_t s_kv[std::max(kBodyLds<D, 8, 1, 2>, kBodyLds<D, 1, 8, 1>) / 2];
  __shared__ float2 s_ml[8 * 64];
  __shared__ int s_others;   // some wave has met infinite or NaN values in an edge block
  TileOf t;
  if (!find_tile<256>(a, t)) return;
  if (threadIdx.x == 0) s_others = 0;   // (the walk's first barrier is before any use)
  Piece p;
  if (t.n_rows - t.first <= 32) {
    if (causal_piece<32, 256>(a, t, p)) extend_body<D, 1, 8, 1, KV8, false>(a, t, p, s_kv, s_ml, nullptr);
  } else {
    if (causal_piece<256, 64>(a, t, p)) extend_body<D, 8, 1, 2, KV8, false>(a, t, p, s_kv, s_ml, &s_others);
  }
}

template <int D, bool KV8>
hipError_t launch_d(const ExtendPlan& p, const ExtendArgs& a, hipStream_t stream) {
  const dim3 grid(a.n_kv_heads, p.tiles, p.n_split);
  if (p.rows == 32) hipLaunchKernelGGL((extend_few_kernel<D, KV8>), grid, dim3(256), 0, stream, a);
  else hipLaunchKernelGGL((extend_many_kernel<D, KV8>), grid, dim3(512), 0, stream, a);
  hipError_t e = hipGetLastError();
  if (e != hipSuccess || p.n_split == 1) return e;
  const int64_t items = (int64_t)a.runs.n_rows * a.n_q_heads;
  const int per = 256 / (D / 4);
  hipLaunchKernelGGL(extend_join_kernel<D>, dim3((unsigned)((items + per - 1) / per)), dim3(256), 0, stream, a, KV8);
  return hipGetLastError();
}

}  // namespace

hipError_t launch_extend(const ExtendPlan& p, int head_dim, bool kv8, const ExtendArgs& a, hipStream_t stream) {
  if (head_dim == 128) return kv8 ? launch_d<128, true>(p, a, stream) : launch_d<128, false>(p, a, stream);
  return kv8 ? launch_d<64, true>(p, a, stream) : launch_d<64, false>(p, a, stream);
}

}  // namespace delta
