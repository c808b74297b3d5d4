// Rotated append of runs of new tokens (Sec. 2, Eq. gqa_projection and kv_update): queries and
// keys turn by their token's position, keys and values go to the paged cache.
//
// Mathematics.  A pair (x, y) of a head turns by the angle p f: (x cos - y sin, y cos + x sin).
// The angle p f of a far position has an fp32 rounding error of 2^-24 p f (0.008 radians at 131072),
// so it is formed in fp64 and reduced there to [-pi, pi] before the fp32 sine and cosine.
//
// Work.  A workgroup takes `tokens` rows (see launch_rope_append).  Wave w finds row w's sequence,
// position and place in the cache, and its lanes the cosines and sines of the row's at most 64
// angles, once for all heads, into LDS.  Then every thread takes units of 16 head elements: two
// 16-byte loads, the rotation, two 16-byte stores (8-byte ones to an e4m3 cache).
//
// Bound: the copy rate for prompts (86423 rows of 40/8 heads into an e4m3 cache, 2.3 GB in 431 us, 5.3
// TB/s, where a plain copy runs at 5.0), launch and the chain of lookups (offset, length, page) for a
// few rows (one row 3.6 us in a graph).
#include "debug_check.h"
#include "runs.h"

namespace delta {
namespace {

constexpr int kThreads = 256;
constexpr int kMaxTokens = kThreads / 64;   // one wave per row

typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));

__device__ __forceinline__ void unpack8(const u32x4& w, float (&x)[8]) {
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    x[2 * i] = __uint_as_float(w[i] << 16);
    x[2 * i + 1] = __uint_as_float(w[i] & 0xffff0000u);
  }
}

// bf16, round to nearest even (NaN stays NaN)
__device__ __forceinline__ u32x4 pack_bf16(const float (&x)[8]) {
  typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
  u32x4 w;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const bf16x2 p = {(__bf16)x[2 * i], (__bf16)x[2 * i + 1]};
    w[i] = __builtin_bit_cast(uint32_t, p);
  }
  return w;
}

// e4m3, round to nearest even, saturated (the conversion instruction turns what is past 448 into
// NaN); NaN stays NaN.
__device__ __forceinline__ u32x2 pack_e4m3(const float (&x)[8], float scale) {
  float y[8];
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const float v = x[i] / scale;
    y[i] = v != v ? v : fminf(fmaxf(v, -448.f), 448.f);
  }
  u32x2 w;
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    int p = __builtin_amdgcn_cvt_pk_fp8_f32(y[4 * i], y[4 * i + 1], 0, false);
    w[i] = __builtin_amdgcn_cvt_pk_fp8_f32(y[4 * i + 2], y[4 * i + 3], p, true);
  }
  return w;
}

template <int D, bool KV8>
__global__ __launch_bounds__(kThreads) void rope_append_kernel(const RopeAppendArgs a, int tokens) {
  constexpr int UPH = D / 16;   // units per head
  const int tid = threadIdx.x, lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int row0 = blockIdx.x * tokens;
  __shared__ float2 s_turn[kMaxTokens][D / 2];   // (cos, sin) of the row's angles
  __shared__ int64_t s_at[kMaxTokens];           // element offset of head 0's cache row; -1: none

  if (wave < tokens) {
    const int row = row0 + wave;
    int64_t at = -1;
    int t = 0;
    const int b = row < a.runs.n_rows ? sequence_of_row(a.runs, row, lane) : -1;
    if (b >= 0) {
      const int begin = run_offset(a.runs, b), end = run_offset(a.runs, b + 1);
      const int s = a.runs.seq_lens[b];
      t = s - (end - row);
      if (s >= end - begin && (s - 1) >> 4 < a.runs.max_pages) {   // (16 * max_pages may pass 32 bits)
        const int page = a.runs.page_table[(size_t)b * a.runs.max_pages + (t >> 4)];
        if (!DELTA_DEBUG || (page >= 0 && (a.n_pages == 0 || page < a.n_pages)))
          at = (int64_t)page * a.page_stride + (t & 15) * D;
      }
    }
    if (lane == 0) s_at[wave] = at;
    if (at >= 0 && lane < a.rotary_dim / 2) {
      const int p = a.positions ? a.positions[row] : t;
      const double angle = (double)p * (double)a.inv_freq[lane];
      constexpr double kTwoPi = 6.283185307179586476925, kTurn = 1.0 / kTwoPi;
      const float r = (float)(angle - kTwoPi * rint(angle * kTurn));
      float sn, cs;
      sincosf(r, &sn, &cs);
      s_turn[wave][lane] = make_float2(cs, sn);
    }
  }
  __syncthreads();

  const int heads = a.n_q_heads + 2 * a.n_kv_heads;
  const int units = heads * UPH;   // of one row
  const int half = a.rotary_dim / 2;
  for (int u = tid; u < tokens * units; u += kThreads) {
    const int i = u / units, rem = u - i * units;
    const int head = rem / UPH, c = rem % UPH;
    const int64_t at = s_at[i];
    if (at < 0) continue;
    const size_t row = row0 + i;
    const bool is_q = head < a.n_q_heads, is_v = head >= a.n_q_heads + a.n_kv_heads;
    const int h = is_q ? head : is_v ? head - a.n_q_heads - a.n_kv_heads : head - a.n_q_heads;
    const uint16_t* src = (is_q ? a.q + row * a.q_stride : is_v ? a.v + row * a.v_stride
                                                                : a.k + row * a.k_stride) + h * D;
    const bool turn = !is_v && 16 * c < a.rotary_dim;
    // the unit's elements: 8 of each half of the rotated part, or 16 in order
    const bool split = turn && !a.interleaved;
    const int e0 = split ? 8 * c : 16 * c, e1 = split ? half + 8 * c : 16 * c + 8;
    float x[8], y[8];
    unpack8(*reinterpret_cast<const u32x4*>(src + e0), x);
    unpack8(*reinterpret_cast<const u32x4*>(src + e1), y);
    if (turn) {
      float2 cs[8];
#pragma unroll
      for (int j = 0; j < 8; ++j) cs[j] = s_turn[i][8 * c + j];
      if (split) {
#pragma unroll
        for (int j = 0; j < 8; ++j) {
          const float p = x[j], r = y[j];
          x[j] = p * cs[j].x - r * cs[j].y;
          y[j] = r * cs[j].x + p * cs[j].y;
        }
      } else {
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          const float p = x[2 * j], r = x[2 * j + 1];
          x[2 * j] = p * cs[j].x - r * cs[j].y;
          x[2 * j + 1] = r * cs[j].x + p * cs[j].y;
          const float p2 = y[2 * j], r2 = y[2 * j + 1];
          y[2 * j] = p2 * cs[j + 4].x - r2 * cs[j + 4].y;
          y[2 * j + 1] = r2 * cs[j + 4].x + p2 * cs[j + 4].y;
        }
      }
    }
    if (is_q) {
      uint16_t* dst = a.q_out + (row * a.n_q_heads + h) * D;
      *reinterpret_cast<u32x4*>(dst + e0) = pack_bf16(x);
      *reinterpret_cast<u32x4*>(dst + e1) = pack_bf16(y);
    } else {
      uint8_t* cache = is_v ? a.v_cache : a.k_cache;
      const size_t off = at + (size_t)h * 16 * D;
      if (KV8) {
        const float* scales = is_v ? a.v_scale : a.k_scale;
        const float scale = scales ? scales[h] : 1.f;
        *reinterpret_cast<u32x2*>(cache + off + e0) = pack_e4m3(x, scale);
        *reinterpret_cast<u32x2*>(cache + off + e1) = pack_e4m3(y, scale);
      } else {
        uint16_t* dst = reinterpret_cast<uint16_t*>(cache) + off;
        *reinterpret_cast<u32x4*>(dst + e0) = pack_bf16(x);
        *reinterpret_cast<u32x4*>(dst + e1) = pack_bf16(y);
      }
    }
  }
}

}  // namespace

hipError_t launch_rope_append(int head_dim, bool kv8, const RopeAppendArgs& a, hipStream_t stream) {
  // One row a workgroup: rows are then looked up and their angles formed in parallel.  Several share
  // one only where a row leaves most of the threads idle and there are rows enough to fill the device.
  // Measured on MI355X, us, one and four rows a workgroup: 64 rows of 32/8 heads 3.9 and 6.2, 1024 6.1
  // and 7.5, 8192 31.6 and 33.0; of 12/2 heads (128 units) 64 rows 3.2 and 3.8, 8192 14.4 and 12.7.
  // (Loading a thread's first units before its row is known: 64 rows of 12/2 heads 4.0 -> 4.5, 9351 of
  // 32/8 35.9 -> 37.8, 86423 of 40/8 431 -> 425; non-temporal loads 456 -> 501 there.)
  const int units = (a.n_q_heads + 2 * a.n_kv_heads) * (head_dim / 16);
  const int tokens = units <= kThreads / 2 && a.runs.n_rows >= 4096 ? kMaxTokens : 1;
  const dim3 grid((a.runs.n_rows + tokens - 1) / tokens), block(kThreads);
  if (head_dim == 128) {
    if (kv8) hipLaunchKernelGGL((rope_append_kernel<128, true>), grid, block, 0, stream, a, tokens);
    else hipLaunchKernelGGL((rope_append_kernel<128, false>), grid, block, 0, stream, a, tokens);
  } else {
    if (kv8) hipLaunchKernelGGL((rope_append_kernel<64, true>), grid, block, 0, stream, a, tokens);
    else hipLaunchKernelGGL((rope_append_kernel<64, false>), grid, block, 0, stream, a, tokens);
  }
  return hipGetLastError();
}

}  // namespace delta
