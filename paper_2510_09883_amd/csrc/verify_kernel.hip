// Which drafted tokens the target's probabilities accept, and the token that follows them.
//
// Mathematics.  Speculative sampling (Leviathan, Kalman and Matias, "Fast inference from transformers via
// speculative decoding", 2023): a draft x drawn from q is accepted with probability min(1, p(x) / q(x)); after
// a rejection the token is to be drawn from max(p - q, 0), normalised, against which the next sibling of the
// tree is tried in the same way (Miao et al., "SpecInfer", 2024).  Nothing is normalised here: the residual r
// keeps its sum R beside it.  All of it is fp64 from fp32 inputs, so that a choice hangs on rounding only where
// a uniform number meets a border to 1e-15.
//
// Work.  n_pieces workgroups take a sequence, and each goes the whole way through the tree by itself: what the
// tests need of the probabilities is one value of the target and one of the drafting model per row, all loaded
// at once, and the rest is comparisons in LDS; rows are tried in ascending order, the current row's next child
// found by a ballot.  (Only where drawn siblings are tried after a rejection does R have to be summed over a
// whole row on the way, by each workgroup for itself.)  Then each sums its piece of the last current row's
// residual, and the one that is done last finds the piece, and in it the token, at which the partial sums pass
// u0 R.  Every sum has a fixed order, so equal calls give equal tokens whichever workgroup is last.
//
// Bound: launch and the chain offsets -> parents -> values for few sequences, HBM for many.
#include <algorithm>

#include "drafts.h"
#include "runs.h"

namespace delta {
namespace {

constexpr int kThreads = 512, kWaves = kThreads / 64;
constexpr int kWindow = 4 * kThreads;            // elements searched at once

__device__ __forceinline__ double wave_sum(double x) {
#pragma unroll
  for (int d = 32; d; d >>= 1) x += __shfl_xor(x, d);
  return x;
}

struct Shared {
  int16_t parent[kMostDrafts];     // -1: never tried
  int32_t token[kMostDrafts];
  float uniform[kMostDrafts], p[kMostDrafts], q[kMostDrafts];
  double left[kMostDrafts];        // R before each rejection at the current row
  double wave[2 * kWaves];
  uint32_t dropped[kMostPiece / 32];   // tokens of the piece that were rejected (draft == null)
  double window[kWindow];
  double sums[2 * kMostPieces];
  int found, last;
};

// The sum over all threads of x, in all of them, in a fixed order.
__device__ __forceinline__ double block_sum(double x, double* s_wave) {
  x = wave_sum(x);
  __syncthreads();
  if ((threadIdx.x & 63) == 0) s_wave[threadIdx.x >> 6] = x;
  __syncthreads();
  double sum = 0;
#pragma unroll
  for (int w = 0; w < kWaves; ++w) sum += s_wave[w];
  return sum;
}

// r after k rejections of drawn drafts (NaN and negative values count as 0).
__device__ __forceinline__ double residual(float p, float q, int k, const double* left) {
  double r = fmax((double)p, 0.0);
  for (int i = 0; i < k; ++i) r = fmax(r - left[i] * (double)q, 0.0);
  return r;
}

__global__ __launch_bounds__(kThreads) void verify_kernel(const VerifyArgs a) {
  __shared__ Shared s;
  const int piece = blockIdx.x, b = blockIdx.y, tid = threadIdx.x, lane = tid & 63;
  const int begin = run_offset(a.runs, b), n = min(run_offset(a.runs, b + 1) - begin, a.max_new);
  int32_t* path = a.path + (size_t)b * a.max_new;
  if (n <= 0) {
    if (piece == 0) {
      for (int i = tid; i < a.max_new; i += kThreads) path[i] = -1;
      if (tid == 0) a.n_path[b] = 0, a.next[b] = -1;
    }
    return;
  }
  const float* target = a.target + (int64_t)begin * a.target_stride;
  const float* draft = a.draft ? a.draft + (int64_t)begin * a.draft_stride : nullptr;

  for (int j = tid; j < n; j += kThreads) {
    int parent = j ? a.parents[begin + j] : -1;
    if (parent < 0 || parent >= j) parent = -1;
    const int x = a.tokens[begin + j];
    const bool some = parent >= 0 && x >= 0 && x < a.vocab;
    s.parent[j] = (int16_t)parent;
    s.token[j] = x;
    s.uniform[j] = a.uniform[begin + j];
    s.p[j] = some ? target[(int64_t)parent * a.target_stride + x] : 0.f;
    s.q[j] = draft ? some ? draft[(int64_t)parent * a.draft_stride + x] : 0.f : 1.f;
  }
  __syncthreads();

  // ---- the way through the tree, the same in all threads
  int cur = 0, count = 1;
  int k = 0;              // rejections at the current row
  int summed = 0;         // of them, those with R known: s.left[0 .. summed] holds R before each and after
  double left = 1.0;      // R, where draft is null
  if (tid == 0) s.left[0] = 1.0;
  if (piece == 0 && tid == 0) path[0] = 0;
  __syncthreads();
  auto sum_left = [&]() {   // R after rejection summed + 1, over the whole row
    const float* p = target + (int64_t)cur * a.target_stride;
    const float* q = draft + (int64_t)cur * a.draft_stride;
    double sum = 0;
    for (int v = tid; v < a.vocab; v += kThreads) sum += residual(p[v], q[v], summed + 1, s.left);
    sum = block_sum(sum, s.wave);
    ++summed;
    if (tid == 0) s.left[summed] = sum;
    __syncthreads();
  };
  for (int c0 = 0; c0 < n; c0 += 64) {
    const int parent = c0 + lane < n ? s.parent[c0 + lane] : -1;
    uint64_t children = __ballot(parent == cur);
    while (children) {
      const int at = __builtin_ctzll(children), j = c0 + at;
      const int x = s.token[j];
      double r, mass;
      if (draft) {
        while (summed < k) sum_left();
        r = residual(s.p[j], s.q[j], k, s.left);
        mass = s.left[k];
      } else {
        r = fmax((double)s.p[j], 0.0);
        mass = left;
        bool again = false;   // a sibling with this token has been rejected
        if (k)
          for (int c = cur & ~63; c <= c0; c += 64)
            again |= __any(c + lane < j && s.parent[c + lane] == cur && s.token[c + lane] == x);
        if (again) r = 0;
      }
      if ((double)s.uniform[j] * (double)s.q[j] * mass < r) {
        if (piece == 0 && tid == 0) path[count] = j;
        cur = j;
        ++count;
        k = summed = 0;
        left = 1.0;
        children = __ballot(parent == cur) & ~((2ull << at) - 1);
      } else {
        ++k;
        if (!draft) left = fmax(left - r, 0.0);
        children &= children - 1;
      }
    }
  }
  if (draft)
    while (summed < k - 1) sum_left();
  if (piece == 0) {
    for (int i = count + tid; i < a.max_new; i += kThreads) path[i] = -1;
    if (tid == 0) a.n_path[b] = count;
  }

  // ---- sums of r and of p over this workgroup's piece
  const float* p = target + (int64_t)cur * a.target_stride;
  const float* q = draft && k ? draft + (int64_t)cur * a.draft_stride : nullptr;
  const int per = (a.vocab + a.n_pieces - 1) / a.n_pieces;
  auto mark_dropped = [&](int v0, int v1) {   // rejected tokens of [v0, v1)
    if (draft || !k) return;
    for (int i = tid; i < (v1 - v0 + 31) / 32; i += kThreads) s.dropped[i] = 0;
    __syncthreads();
    for (int j = cur + 1 + tid; j < n; j += kThreads) {
      const int x = s.token[j];
      if (s.parent[j] == cur && x >= v0 && x < v1) atomicOr(&s.dropped[(x - v0) >> 5], 1u << ((x - v0) & 31));
    }
    __syncthreads();
  };
  auto r_of = [&](int v, int v0) {
    if (draft) return residual(p[v], q ? q[v] : 0.f, k, s.left);
    const double r = fmax((double)p[v], 0.0);
    return k && (s.dropped[(v - v0) >> 5] >> ((v - v0) & 31) & 1) ? 0.0 : r;
  };
  {
    const int v0 = min(piece * per, a.vocab), v1 = min(v0 + per, a.vocab);
    mark_dropped(v0, v1);
    double sum_r = 0, sum_p = 0;
    for (int v = v0 + tid; v < v1; v += kThreads) {
      sum_r += r_of(v, v0);
      sum_p += fmax((double)p[v], 0.0);
    }
    sum_r = block_sum(sum_r, s.wave);
    sum_p = block_sum(sum_p, s.wave);
    if (tid == 0) {
      double* out = a.state[b].sums[piece];
      __hip_atomic_store(out, sum_r, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
      __hip_atomic_store(out + 1, sum_p, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
      int32_t* counter = &a.state[b].arrived;
      const int arrived = __hip_atomic_fetch_add(counter, 1, __ATOMIC_ACQ_REL, __HIP_MEMORY_SCOPE_AGENT);
      s.last = arrived == a.n_pieces - 1;
      if (s.last) __hip_atomic_store(counter, 0, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);   // ready for the next call
    }
    __syncthreads();
    if (!s.last) return;
  }

  // ---- the last one: the piece in which the partial sums pass u0 times the whole
  if (tid < 2 * a.n_pieces)
    s.sums[tid] = __hip_atomic_load(&a.state[b].sums[0][0] + tid, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
  __syncthreads();
  double total = 0, total_p = 0;
  for (int i = 0; i < a.n_pieces; ++i) total += s.sums[2 * i], total_p += s.sums[2 * i + 1];
  const bool use_p = !(total > 0);
  if (use_p) total = total_p;
  if (!(total > 0)) {
    if (tid == 0) a.next[b] = -1;
    return;
  }
  const double goal = (double)s.uniform[0] * total;
  double before = 0, cum = 0;
  int where = 0;
  for (int i = 0; i < a.n_pieces; ++i) {
    const double x = s.sums[2 * i + use_p];
    if (x > 0) {
      where = i;
      before = cum;
      if (cum + x > goal) break;
    }
    cum += x;
  }
  const int v0 = min(where * per, a.vocab), v1 = min(v0 + per, a.vocab);
  mark_dropped(v0, v1);

  // ---- the token: windows of the piece, four elements in a row per thread
  int last_some = v0;   // the last token with r > 0 so far
  for (int w0 = v0; w0 < v1; w0 += kWindow) {
    __syncthreads();
    if (tid == 0) s.found = INT32_MAX, s.last = -1;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int v = w0 + i * kThreads + tid;
      s.window[i * kThreads + tid] = v >= v1 ? 0.0 : use_p ? fmax((double)p[v], 0.0) : r_of(v, v0);
    }
    __syncthreads();
    double x[4], own = 0;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      x[i] = s.window[4 * tid + i];
      own += x[i];
    }
    double incl = own;
#pragma unroll
    for (int d = 1; d < 64; d <<= 1) {
      const double y = __shfl_up(incl, d);
      if (lane >= d) incl += y;
    }
    if (lane == 63) s.wave[tid >> 6] = incl;
    __syncthreads();
    double waves = 0, all = 0;
#pragma unroll
    for (int w = 0; w < kWaves; ++w) {
      if (w < tid >> 6) waves += s.wave[w];
      all += s.wave[w];
    }
    double excl = __shfl_up(incl, 1);
    if (lane == 0) excl = 0;
    if (own > 0 && before + (waves + incl) > goal) {
      double c = before + (waves + excl);
      int v = -1;
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        if (x[i] > 0 && (v < 0 || !(c > goal))) v = w0 + 4 * tid + i;   // (the first that passes, else the last > 0)
        c += x[i];
      }
      atomicMin(&s.found, v);
    }
    if (own > 0) {
      int v = 0;
#pragma unroll
      for (int i = 0; i < 4; ++i)
        if (x[i] > 0) v = w0 + 4 * tid + i;
      atomicMax(&s.last, v);
    }
    __syncthreads();
    if (s.found != INT32_MAX) {
      if (tid == 0) a.next[b] = s.found;
      return;
    }
    if (s.last >= 0) last_some = s.last;
    before += all;
  }
  if (tid == 0) a.next[b] = last_some;
}

}  // namespace

hipError_t launch_verify(const VerifyArgs& a, hipStream_t stream) {
  hipLaunchKernelGGL(verify_kernel, dim3(a.n_pieces, a.runs.batch), dim3(kThreads), 0, stream, a);
  return hipGetLastError();
}

}  // namespace delta
