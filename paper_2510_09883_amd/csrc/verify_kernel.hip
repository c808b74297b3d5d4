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
// whole row on the way, by each workgroup for itself.)  Then each wave sums its part of the last current row's
// residual.  A second launch finds the part, and in it the token, at which the partial sums pass u0 R.  Every sum
// has a fixed order, so equal calls give equal tokens.
//
// Bound (medians of 200 dispatches): latencies, of launches and of the chains offsets -> parents -> values -> row and sums -> row (one tree of 16
// chosen drafts, 151936 tokens: 5.6 us and 4.0); then the reads of the rows (64 chains of drawn drafts, of which 41 end in a
// rejection and read the drafts' row too, 64 MB: 16.4 us, 3.9 TB/s, and 4.6).  A sum of R over 151936 tokens takes 13 us (16
// trees of 8 rows, up to three drawn siblings: 33 and 4.8).  Measured for the chains, both launches in a graph: finding the token by LDS atomics of all threads on
// one word 38 us, by ballots 31; with parts that are whole rounds of 16 bytes a lane, where nearly half of a part was
// read 4 bytes a lane before, 25.  That the last of a sequence's workgroups to arrive at a counter picks the token was
// no faster than a second launch (38 us for both), and 208 with release and acquire at the counter.
#include <algorithm>

#include "drafts.h"
#include "runs.h"

namespace delta {
namespace {

constexpr int kWaves = kVerifyWaves, kThreads = 64 * kWaves;
typedef float f32x4 __attribute__((ext_vector_type(4)));

// x of another lane of the row, or of another row (0 where there is none): see wave_incl_scan.
template <int CTRL, int ROWS>
__device__ __forceinline__ double moved(double x) {
  const uint64_t w = __builtin_bit_cast(uint64_t, x);
  const uint32_t lo = __builtin_amdgcn_update_dpp(0, (int)(uint32_t)w, CTRL, ROWS, 0xf, false);
  const uint32_t hi = __builtin_amdgcn_update_dpp(0, (int)(uint32_t)(w >> 32), CTRL, ROWS, 0xf, false);
  return __builtin_bit_cast(double, (uint64_t)hi << 32 | lo);
}
// Inclusive prefix sums over the 64 lanes.
__device__ __forceinline__ double wave_scan(double x) {
  x += moved<0x111, 0xf>(x);
  x += moved<0x112, 0xf>(x);
  x += moved<0x114, 0xf>(x);
  x += moved<0x118, 0xf>(x);
  x += moved<0x142, 0xa>(x);
  x += moved<0x143, 0xc>(x);
  return x;
}
__device__ __forceinline__ double lane_of(double x, int lane) {
  const uint64_t w = __builtin_bit_cast(uint64_t, x);
  const uint32_t lo = __builtin_amdgcn_readlane((int)(uint32_t)w, lane);
  const uint32_t hi = __builtin_amdgcn_readlane((int)(uint32_t)(w >> 32), lane);
  return __builtin_bit_cast(double, (uint64_t)hi << 32 | lo);
}
__device__ __forceinline__ double wave_sum(double x) { return lane_of(wave_scan(x), 63); }

struct Shared {
  int16_t parent[kMostDrafts];     // -1: never tried
  int32_t token[kMostDrafts];
  float uniform[kMostDrafts], p[kMostDrafts], q[kMostDrafts];
  double wave[kWaves];
  uint32_t dropped[kMostPiece / 32];   // tokens of the piece that were rejected (draft == null)
};

struct SharedPick {
  double wave[kWaves], before;
  double part[kMostPieces * kWaves];   // sums of p, where they are needed
  uint32_t dropped[kMostPiece / 32];
  double window[kMostPart];
  int past[kWaves], some[kWaves];
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

// Inclusive prefix sums over the threads, what stands before the thread, and the sum, each in a fixed order.
__device__ __forceinline__ double block_scan(double x, double* s_wave, double* incl, double* excl) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const double sum = wave_scan(x);
  __syncthreads();
  if (lane == 63) s_wave[wave] = sum;
  __syncthreads();
  double waves = 0, all = 0;
#pragma unroll
  for (int w = 0; w < kWaves; ++w) {
    if (w < wave) waves += s_wave[w];
    all += s_wave[w];
  }
  *incl = waves + sum;
  const double before = __shfl_up(sum, 1);
  *excl = waves + (lane ? before : 0.0);
  return all;
}

// f(v, p[v], q[v]) for the elements first .. end - 1, which THREADS threads share, t the caller's number among them.
// In full rounds a thread has 16 elements of each row under way; 16 bytes at once where the rows are aligned to them
// (first is a multiple of 4).
template <int THREADS, class F>
__device__ __forceinline__ void for_row(const float* p, const float* q, int first, int end, int t, F f) {
  constexpr int kRound = 16 * THREADS;
  int v = first;
  if (((reinterpret_cast<uintptr_t>(p) | reinterpret_cast<uintptr_t>(q)) & 15) == 0) {
    for (; v + kRound <= end; v += kRound) {
      f32x4 x[4], y[4];
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const int at = v + 4 * (i * THREADS + t);
        x[i] = *reinterpret_cast<const f32x4*>(p + at);
        if (q) y[i] = *reinterpret_cast<const f32x4*>(q + at);
        else y[i] = f32x4{0.f, 0.f, 0.f, 0.f};
      }
#pragma unroll
      for (int i = 0; i < 4; ++i)
#pragma unroll
        for (int c = 0; c < 4; ++c) f(v + 4 * (i * THREADS + t) + c, x[i][c], y[i][c]);
    }
  } else {
    for (; v + kRound <= end; v += kRound) {
      float x[16], y[16];
#pragma unroll
      for (int i = 0; i < 16; ++i) {
        x[i] = p[v + i * THREADS + t];
        y[i] = q ? q[v + i * THREADS + t] : 0.f;
      }
#pragma unroll
      for (int i = 0; i < 16; ++i) f(v + i * THREADS + t, x[i], y[i]);
    }
  }
  if (v >= end) return;
  float x[16], y[16];
#pragma unroll
  for (int i = 0; i < 16; ++i) {   // (past the end: the last element again, not counted)
    const int at = min(v + i * THREADS + t, end - 1);
    x[i] = p[at];
    y[i] = q ? q[at] : 0.f;
  }
#pragma unroll
  for (int i = 0; i < 16; ++i)
    if (v + i * THREADS + t < end) f(v + i * THREADS + t, x[i], y[i]);
}

// A probability; negative and NaN ones count as 0.
__device__ __forceinline__ double mass_of(float x) { return fmaxf(x, 0.f); }

// r after rejections of drawn drafts, S the sum of R before each of them: as q and R are not negative,
// max(max(p - R0 q, 0) - R1 q, 0) = max(p - (R0 + R1) q, 0), and so on.
__device__ __forceinline__ double residual(float p, float q, double S) { return fmax(mass_of(p) - S * mass_of(q), 0.0); }

// The current row's probabilities after k rejections, in pieces and waves' parts of them.
struct Row {
  const float *p, *q;          // q: null where it is not needed
  int vocab, part, per;        // elements of a part and of a piece
  int k;
  bool drawn;
  double S;                    // of drawn drafts: see residual
  uint32_t* dropped;           // LDS: rejected tokens of a piece, if they were not drawn

  __device__ __forceinline__ Row(const VerifyArgs& a, int begin, int cur, int k, double S, uint32_t* dropped)
      : p(a.target + (int64_t)(begin + cur) * a.target_stride),
        q(a.draft && k ? a.draft + (int64_t)(begin + cur) * a.draft_stride : nullptr),
        vocab(a.vocab), k(k), drawn(a.draft != nullptr), S(S), dropped(dropped) {
    part = a.part;
    per = part * kWaves;
  }
  __device__ __forceinline__ int begin_of(int i) const { return min(i * part, vocab); }
  __device__ __forceinline__ int end_of(int i) const { return min((i + 1) * part, vocab); }
  // Notes the rejected tokens from v0 on: tokens of rows cur + 1 .. n - 1 whose parent is cur.
  template <class Parent, class Token>
  __device__ __forceinline__ void mark_dropped(int v0, int cur, int n, Parent parent, Token token) const {
    if (drawn || !k) return;
    const int v1 = min(v0 + per, vocab);
    for (int i = threadIdx.x; i < (per + 31) / 32; i += kThreads) dropped[i] = 0;
    __syncthreads();
    for (int j = cur + 1 + threadIdx.x; j < n; j += kThreads)
      if (parent(j) == cur) {
        const int x = token(j);
        if (x >= v0 && x < v1) atomicOr(&dropped[(x - v0) >> 5], 1u << ((x - v0) & 31));
      }
    __syncthreads();
  }
  // r of element v of the piece from v0 on
  __device__ __forceinline__ double r_of(int v, float x, float y, int v0) const {
    if (drawn) return residual(x, y, S);
    return k && (dropped[(v - v0) >> 5] >> ((v - v0) & 31) & 1) ? 0.0 : mass_of(x);
  }
};

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
    s.q[j] = draft ? some ? fmaxf(draft[(int64_t)parent * a.draft_stride + x], 0.f) : 0.f : 1.f;
  }
  __syncthreads();

  // ---- the way through the tree, the same in all threads
  int cur = 0, count = 1;
  int k = 0;              // rejections at the current row
  double R = 1.0, S = 0.0;   // r's sum, and of drawn drafts the sum of R before each rejection
  bool known = true;         // (R is formed when a test needs it)
  if (piece == 0 && tid == 0) path[0] = 0;
  auto sum_row = [&]() {     // R, over the whole row
    const float* p = target + (int64_t)cur * a.target_stride;
    const float* q = draft + (int64_t)cur * a.draft_stride;
    double sum = 0;
    for_row<kThreads>(p, q, 0, a.vocab, tid, [&](int, float x, float y) { sum += residual(x, y, S); });
    R = block_sum(sum, s.wave);
    known = true;
  };
  for (int c0 = 0; c0 < n; c0 += 64) {
    const int parent = c0 + lane < n ? s.parent[c0 + lane] : -1;
    uint64_t children = __ballot(parent == cur);
    while (children) {
      const int at = __builtin_ctzll(children), j = c0 + at;
      const int x = s.token[j];
      double r;
      if (draft) {
        if (!known) sum_row();
        r = residual(s.p[j], s.q[j], S);
      } else {
        r = mass_of(s.p[j]);
        bool again = false;   // a sibling with this token has been rejected
        if (k)
          for (int c = cur & ~63; c <= c0; c += 64)
            again |= __any(c + lane < j && s.parent[c + lane] == cur && s.token[c + lane] == x);
        if (again) r = 0;
      }
      if ((double)s.uniform[j] * (double)s.q[j] * R < r) {
        if (piece == 0 && tid == 0) path[count] = j;
        cur = j;
        ++count;
        k = 0;
        R = 1.0, S = 0.0;
        known = true;
        children = __ballot(parent == cur) & ~((2ull << at) - 1);
      } else {
        ++k;
        if (draft) {
          S += R;
          known = false;
        } else {
          R = fmax(R - r, 0.0);
        }
        children &= children - 1;
      }
    }
  }
  if (piece == 0) {
    for (int i = count + tid; i < a.max_new; i += kThreads) path[i] = -1;
    if (tid == 0) a.n_path[b] = count;
  }

  // ---- the sum of r over this workgroup's piece, a part of it by each wave
  const Row row(a, begin, cur, k, S, s.dropped);
  const int v0 = piece * row.per, mine = piece * kWaves + (tid >> 6);
  row.mark_dropped(v0, cur, n, [&](int j) { return (int)s.parent[j]; }, [&](int j) { return s.token[j]; });
  double sum = 0;
  for_row<64>(row.p, row.q, row.begin_of(mine), row.end_of(mine), lane, [&](int v, float x, float y) { sum += row.r_of(v, x, y, v0); });
  sum = wave_sum(sum);
  VerifyState& state = a.state[b];
  if (lane == 0) state.sums[mine] = sum;
  if (piece == 0 && tid == 0) state.cur = cur, state.k = k, state.S = S;
}

// The token after the accepted rows: the part, and in it the element, at which the partial sums of r pass u0 times
// the whole.  A workgroup takes a sequence.
__global__ __launch_bounds__(kThreads) void verify_pick_kernel(const VerifyArgs a) {
  __shared__ SharedPick s;
  const int b = blockIdx.x, tid = threadIdx.x, lane = tid & 63;
  const int n_parts = a.n_pieces * kWaves;
  const VerifyState& state = a.state[b];
  // (loaded together; of an empty run they are anything)
  const int begin = run_offset(a.runs, b), n = min(run_offset(a.runs, b + 1) - begin, a.max_new);
  const int cur = state.cur, k = state.k;
  const double S = state.S;
  double part_sum = tid < n_parts ? state.sums[tid] : 0.0;
  if (n <= 0) return;
  const double u0 = a.uniform[begin];
  const Row row(a, begin, cur, k, S, s.dropped);
  double incl, excl;
  double total = block_scan(part_sum, s.wave, &incl, &excl);
  const bool use_p = !(total > 0);
  if (use_p) {   // (nothing is left: p takes the place of r)
    for (int i = tid >> 6; i < n_parts; i += kWaves) {
      double sum = 0;
      for_row<64>(row.p, nullptr, row.begin_of(i), row.end_of(i), lane, [&](int, float x, float) { sum += mass_of(x); });
      sum = wave_sum(sum);
      if (lane == 0) s.part[i] = sum;
    }
    __syncthreads();
    part_sum = tid < n_parts ? s.part[tid] : 0.0;
    total = block_scan(part_sum, s.wave, &incl, &excl);
    if (!(total > 0)) {
      if (tid == 0) a.next[b] = -1;
      return;
    }
  }
  const double goal = u0 * total;
  // the thread whose own numbers pass the goal first, or else the last that has any
  auto first_past = [&](double before, double own) {
    const uint64_t some = __ballot(own > 0), past = __ballot(own > 0 && before + incl > goal);
    if (lane == 0) {
      s.past[tid >> 6] = past ? tid + __builtin_ctzll(past) : INT32_MAX;
      s.some[tid >> 6] = some ? tid + 63 - __builtin_clzll(some) : -1;
    }
    __syncthreads();
    int found = INT32_MAX, last = -1;
#pragma unroll
    for (int w = 0; w < kWaves; ++w) {
      found = min(found, s.past[w]);
      last = max(last, s.some[w]);
    }
    return found != INT32_MAX ? found : last;
  };
  const int where = first_past(0, part_sum);
  if (tid == where) s.before = excl;

  // ---- the token: the part's elements, four in a row per thread
  const int v0 = row.begin_of(where), v1 = row.end_of(where), piece0 = where / kWaves * row.per;
  static_assert(kMostPart == 4 * kThreads, "four elements a thread");
  float x[4], y[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const int v = min(v0 + i * kThreads + tid, v1 - 1);
    x[i] = row.p[v];
    y[i] = row.q && !use_p ? row.q[v] : 0.f;
  }
  row.mark_dropped(piece0, cur, n, [&](int j) { return a.parents[begin + j]; }, [&](int j) { return a.tokens[begin + j]; });
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const int v = v0 + i * kThreads + tid;
    s.window[i * kThreads + tid] = v >= v1 ? 0.0 : use_p ? mass_of(x[i]) : row.r_of(v, x[i], y[i], piece0);
  }
  __syncthreads();
  const double before = s.before;
  double r[4], own = 0;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    r[i] = s.window[4 * tid + i];
    own += r[i];
  }
  block_scan(own, s.wave, &incl, &excl);
  if (tid == first_past(before, own)) {
    double c = before + excl;
    int v = 0;
    bool some = false;
#pragma unroll
    for (int i = 0; i < 4; ++i) {   // the first that passes, else the last > 0
      if (r[i] > 0 && (!some || !(c > goal))) v = 4 * tid + i, some = true;
      c += r[i];
    }
    a.next[b] = v0 + v;
  }
}

}  // namespace

hipError_t launch_verify(const VerifyArgs& a, hipStream_t stream) {
  hipLaunchKernelGGL(verify_kernel, dim3(a.n_pieces, a.runs.batch), dim3(kThreads), 0, stream, a);
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;
  hipLaunchKernelGGL(verify_pick_kernel, dim3(a.runs.batch), dim3(kThreads), 0, stream, a);
  return hipGetLastError();
}

}  // namespace delta
