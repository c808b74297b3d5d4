// Causal attention of runs of new tokens over the paged cache (Sec. 2, Eq. gqa_attention, for more
// than one query token of a sequence).
//
// Mathematics.  A row is one (new token, query head) pair.  out = sum_t p_t v_t / sum_t p_t over the
// tokens t the row sees, p_t = 2^(s_t - m), s_t the scaled score in the log2 domain, m the running
// maximum: one pass over the keys, the sums rescaled when the maximum rises (Milakov and Gimelshein,
// "Online normalizer calculation for softmax", 2018).
//
// Work.  The rows of a run that share a KV head (token-major, the group's query heads next to each
// other) are cut into tiles; a workgroup takes a tile, and one of n_split pieces of the keys that
// the tile's last row sees (extend_api.cpp decides the cut).  A wave holds 32 rows and takes 32*KT
// keys of a block; WR waves stand along the rows, WK along the keys.  Two kernels:
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
// Per 32 keys and wave:
//   * S^T = K Q^T by v_mfma_f32_32x32x16_bf16 with A = 32 keys, B = the 32 rows' queries (in
//     registers throughout).  Lane (h, n) = (lane / 32, lane % 32) gets row n's scores of keys
//     8*(i/4) + 4*h + i%4, i = 0 .. 15: a row lives in two lanes, so that its maximum and sum are
//     formed in registers and one swap of the wave's halves.
//   * O^T = V^T P^T by the same instruction.  Its B operand wants row n's probabilities of 8 keys
//     in lane (h, n), which is what the lane holds: keys 16*s + 4*h + {0..3} and 16*s + 8 + 4*h +
//     {0..3}.  The order of the keys in a contraction is free as long as A has the same one: V
//     comes from LDS by ds_read_b64_tr_b16, which hands 4 consecutive keys of one element to a
//     lane, once for each four.  No probability changes its lane.
//
// LDS layouts: K rows with their 16-byte pieces permuted by the row (16 lanes reading one piece of
// 16 rows touch all banks), V rows with their 64-byte pieces permuted by the row (the four rows of
// a transposing read do).  The counters show no bank conflict.
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
#include <algorithm>

#include "attn_tile.h"
#include "debug_check.h"
#include "runs.h"

namespace delta {
namespace {

typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef __attribute__((address_space(3))) i16x4 lds_i16x4;

// Element offset of 8-element piece c of row r of the K block.
template <int D>
__device__ __forceinline__ int k_at(int r, int c) {
  return r * D + 8 * (c ^ (D == 128 ? r & 15 : (r >> 1) & 7));
}
// Element offset of element e of row r of the V block.
template <int D>
__device__ __forceinline__ int v_at(int r, int e) {
  return r * D + (e ^ (D == 128 ? (r & 3) << 5 : ((r >> 1) & 1) << 5));
}

// Infinite and NaN values among two bf16 (all exponent bits set) or four e4m3 (NaN: all bits but the
// sign's set): `seen` gathers what tells of them, has_others reads it, without_others makes them 0.
template <bool KV8>
__device__ __forceinline__ void look_for_others(uint32_t w, uint32_t& seen) {
  typedef uint16_t u16x2 __attribute__((ext_vector_type(2)));
  if (KV8) seen |= (w & 0x7f7f7f7fu) + 0x01010101u;
  else
    seen = __builtin_bit_cast(uint32_t, __builtin_elementwise_max(__builtin_bit_cast(u16x2, seen),
                                                                  __builtin_bit_cast(u16x2, w & 0x7fff7fffu)));
}
template <bool KV8>
__device__ __forceinline__ bool has_others(uint32_t seen) {
  return KV8 ? (seen & 0x80808080u) != 0 : (seen >> 16) >= 0x7f80u || (seen & 0xffffu) >= 0x7f80u;
}
template <bool KV8>
__device__ __forceinline__ uint32_t without_others(uint32_t w) {
  if (KV8) return w & ~(((((w & 0x7f7f7f7fu) + 0x01010101u) & 0x80808080u) >> 7) * 0xffu);
  return w & ~(((((w & 0x7f807f80u) + 0x00800080u) & 0x80008000u) >> 15) * 0xffffu);
}

// Four outputs, scaled and divided by the softmax sum, as bf16; a row that sees no key (l = 0) gets
// zeros.  (Divided: a product by 1 / l has a rounding more, which moves quotients half way between
// two bf16 values, as equal weights give.)
__device__ __forceinline__ u32x2 pack_outputs(const f32x4& x, float scale, float l) {
  u32x2 w;
#pragma unroll
  for (int k = 0; k < 2; ++k) {
    const float a = x[2 * k] * scale, b = x[2 * k + 1] * scale;
    const bf16x2 p = {(__bf16)(l == 0.f ? 0.f : a / l), (__bf16)(l == 0.f ? 0.f : b / l)};
    w[k] = __builtin_bit_cast(uint32_t, p);
  }
  return w;
}

// What a workgroup knows of its tile.
struct TileOf {
  int b;         // the sequence
  int begin;     // first row of its run
  int n_rows;    // (token, query head) rows of its run
  int n_new;     // tokens of its run
  int first;     // first of the rows that the tile takes
  int s_b;       // tokens of the sequence
};

// LDS of a body, in bytes: K and V of the blocks, later the outputs of the waves along the keys.
template <int D, int WR, int WK, int KT>
constexpr int kBodyLds = std::max(2 * (WR == 1 ? 1 : 2) * 32 * KT * WK * D * 2, WK > 1 ? WK * 64 * D / 2 * 4 : 0);

template <int D, int WR, int WK, int KT, bool KV8>
__device__ __forceinline__ void extend_body(const ExtendArgs& a, const TileOf& t, uint16_t* s_kv, float2* s_ml,
                                            int* s_others) {
  constexpr int NW = WR * WK, T = 64 * NW;
  constexpr int BM = 32 * WR;           // rows of a tile
  constexpr int BK = 32 * KT;           // keys a wave takes of a block
  constexpr int BN = BK * WK;           // keys of a block
  constexpr int NK = D / 16;            // MFMA steps of a score tile
  constexpr int ND = D / 32;            // 32-element parts of an output row
  constexpr int EB = KV8 ? 1 : 2;       // bytes of a cache element
  constexpr int CPR = D * EB / 16;      // 16-byte pieces of a cache row
  constexpr int kPieces = BN * CPR;     // of a block, of K and of V
  constexpr int NL = (kPieces + T - 1) / T;   // loads per thread and block (the last waves may have none)
  constexpr int RPW = 64 / CPR;         // rows of a wave-wide load
  static_assert(kPieces % 64 == 0 && 16 % RPW == 0, "whole loads, each inside one page");
  const int lane = threadIdx.x & 63;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int wr = wave % WR, wk = wave / WR;
  const int n = lane & 31, h = lane >> 5;
  const int g = blockIdx.x, split = blockIdx.z;
  const int Hq = a.n_q_heads, G = Hq / a.n_kv_heads;

  // Waves that share no rows share no keys either: each brings its own keys to its own LDS, without
  // barriers, and needs one buffer of it.
  constexpr bool kOwnKeys = WR == 1;
  constexpr int kBuffers = kOwnKeys ? 1 : 2;
  constexpr int kBlock = BN * D;        // elements of a K or V block
  const int b = t.b, n_new = t.n_new, s_b = t.s_b, n_tile_rows = t.n_rows, begin = t.begin;
  // this lane's row: token j of the run, query head g * G + head
  const int r0 = t.first + 32 * wr;
  const int r = min(r0 + n, n_tile_rows - 1);
  const bool real = r0 + n < n_tile_rows;
  const bool active = r0 < n_tile_rows;                               // some row of the wave is
  const int j = r / G, head = g * G + (r - j * G);
  const size_t out_row = (size_t)(begin + j) * Hq + head;
  const int lim = max(0, s_b - n_new + j + 1);                        // keys the row sees
  auto lim_of = [&](int row) { return max(0, s_b - n_new + min(row, n_tile_rows - 1) / G + 1); };
  const int lim_lo = lim_of(r0), lim_hi = lim_of(r0 + 31);            // of the wave's rows

  const int n_blocks = (lim_of(t.first + BM - 1) + BN - 1) / BN;
  // pieces of one length whatever the sequence's: a short sequence has fewer
  const int per_split = a.split_keys / BN;
  const int n_valid = max(1, (n_blocks + per_split - 1) / per_split);
  if (split >= n_valid) return;
  const int blk0 = split * per_split, blk1 = min(n_blocks, blk0 + per_split);

  const float scale = KV8 && a.k_scale ? a.scale_log2 * a.k_scale[g] : a.scale_log2;
  bf16x8 q[NK];
#pragma unroll
  for (int ks = 0; ks < NK; ++ks)
    q[ks] = __builtin_bit_cast(bf16x8, *reinterpret_cast<const u32x4*>(a.q + out_row * D + 16 * ks + 8 * h));
  // they are waited for here: a wait for their first use, inside the loop, would also wait for the
  // loads of the next block in every round
#pragma unroll
  for (int ks = 0; ks < NK; ++ks) asm volatile("" : "+v"(q[ks]));

  float m = kNegInfF, l = 0.f;
  f32x16 o[ND];
#pragma unroll
  for (int i = 0; i < ND; ++i) o[i] = f32x16{};

  // ---- blocks: pages of the next 64 (one per lane), loads, LDS ------------------------------
  const int32_t* table = a.runs.page_table + (size_t)b * a.runs.max_pages;
  const int last_page = max(0, (s_b - 1) >> 4);
  int page_base = blk0 * BN / 16;
  int pages = 0;
  auto list_pages = [&](int base) {
    pages = checked_page(table[min(base + lane, last_page)], a.n_pages, a.status);
    page_base = base;
  };
  u32x4 kr[NL], vr[NL];
  // the wave's first row of load i, in the block
  auto row_of = [&](int i) { return kOwnKeys ? wk * BK + i * RPW : (i * NW + wave) * RPW; };
  const uint32_t lane16 = 16 * lane;
  auto load = [&](int blk) {
    const int first = blk * BN / 16;
    if (first + BN / 16 > page_base + 64) list_pages(first);
#pragma unroll
    for (int i = 0; i < NL; ++i) {
      const int row = row_of(i);
      if (kPieces % T && row >= BN) break;
      const int page = __builtin_amdgcn_readlane(pages, first + row / 16 - page_base);
      // (uniform: scalar arithmetic, and the lane's offset is the loads' own)
      const size_t at = ((size_t)(uint32_t)page * (uint32_t)a.page_stride + (uint32_t)((g * 16 + row % 16) * D)) * EB;
      const u32x4* kp = reinterpret_cast<const u32x4*>(a.k_cache + at + lane16);
      const u32x4* vp = reinterpret_cast<const u32x4*>(a.v_cache + at + lane16);
      kr[i] = kOwnKeys ? __builtin_nontemporal_load(kp) : *kp;
      vr[i] = kOwnKeys ? __builtin_nontemporal_load(vp) : *vp;
    }
  };
  // Where some rows of the tile do not see all keys of a block (an edge block; only there do keys lie
  // past the sequence), 0 times a value that is infinite or NaN would reach rows that do not see its
  // token: such values go to LDS as 0, and the rows that do see them get them at the end.  (Looking for
  // them takes 0.2 us of 7.2 where every block is an edge block, 8 short sequences, else no time seen;
  // replacing them without looking took 0.6.)
  const int lim_first = lim_of(t.first);
  bool others = false;   // the wave has met such values
  auto store = [&](int blk, int buf) {
    uint16_t* sk = s_kv + buf * 2 * kBlock;
    uint16_t* sv = sk + kBlock;
    if ((blk + 1) * BN > lim_first) {
      uint32_t seen = 0;
#pragma unroll
      for (int i = 0; i < NL; ++i) {
        if (kPieces % T && row_of(i) >= BN) break;
        if (blk * BN + row_of(i) + lane / CPR >= s_b) vr[i] = u32x4{0u, 0u, 0u, 0u};
#pragma unroll
        for (int w = 0; w < 4; ++w) look_for_others<KV8>(vr[i][w], seen);
      }
      if (__any(has_others<KV8>(seen))) {
        others = true;
#pragma unroll
        for (int i = 0; i < NL; ++i) {
          if (kPieces % T && row_of(i) >= BN) break;
#pragma unroll
          for (int w = 0; w < 4; ++w) vr[i][w] = without_others<KV8>(vr[i][w]);
        }
      }
    }
#pragma unroll
    for (int i = 0; i < NL; ++i) {
      const int row = row_of(i) + lane / CPR, c = lane % CPR;
      if (kPieces % T && row >= BN) break;
      if constexpr (KV8) {
#pragma unroll
        for (int half = 0; half < 2; ++half) {
          u32x4 wk, wv;
#pragma unroll
          for (int w = 0; w < 2; ++w) {
            wk[2 * w] = e4m3x2_to_bf16x2<false>(kr[i][2 * half + w]);
            wk[2 * w + 1] = e4m3x2_to_bf16x2<true>(kr[i][2 * half + w]);
            wv[2 * w] = e4m3x2_to_bf16x2<false>(vr[i][2 * half + w]);
            wv[2 * w + 1] = e4m3x2_to_bf16x2<true>(vr[i][2 * half + w]);
          }
          *reinterpret_cast<u32x4*>(sk + k_at<D>(row, 2 * c + half)) = wk;
          *reinterpret_cast<u32x4*>(sv + v_at<D>(row, 16 * c + 8 * half)) = wv;
        }
      } else {
        *reinterpret_cast<u32x4*>(sk + k_at<D>(row, c)) = kr[i];
        *reinterpret_cast<u32x4*>(sv + v_at<D>(row, 8 * c)) = vr[i];
      }
    }
  };

  auto attend = [&](int blk, int buf) {
    const int key0 = blk * BN + wk * BK;   // the wave's first key
    if ((WR > 1 && !active) || key0 >= lim_hi) return;
    const uint16_t* sk = s_kv + buf * 2 * kBlock + wk * BK * D;
    const uint16_t* sv = s_kv + buf * 2 * kBlock + kBlock + wk * BK * D;
    f32x16 s[KT];
#pragma unroll
    for (int kt = 0; kt < KT; ++kt) {
      s[kt] = f32x16{};
#pragma unroll
      for (int ks = 0; ks < NK; ++ks) {
        const bf16x8 ka = __builtin_bit_cast(
            bf16x8, *reinterpret_cast<const u32x4*>(sk + k_at<D>(32 * kt + n, 2 * ks + h)));
        s[kt] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(ka, q[ks], s[kt], 0, 0, 0);
      }
    }
    {
// a scaled score is rounded before the maximum and the difference see it: contracted into the
// difference's fma, the maximum's own rounding error would be left in the exponent
#pragma clang fp contract(off)
#pragma unroll
      for (int kt = 0; kt < KT; ++kt) s[kt] *= scale;
      if (key0 + BK > lim_lo) {   // some row of the wave does not see all of these keys
#pragma unroll
        for (int kt = 0; kt < KT; ++kt)
#pragma unroll
          for (int i = 0; i < 16; ++i) {
            const int key = key0 + 32 * kt + 8 * (i / 4) + 4 * h + i % 4;
            s[kt][i] = key < lim ? s[kt][i] : kNegInfF;
          }
      }
      float mx = s[0][0];
#pragma unroll
      for (int kt = 0; kt < KT; ++kt)
#pragma unroll
        for (int i = 0; i < 16; ++i) mx = fmaxf(mx, s[kt][i]);
      mx = max_xor32(mx);
      if (__any(mx > m)) {
        const float m_new = fmaxf(m, mx);
        const float alpha = __builtin_amdgcn_exp2f(m - (m_new == kNegInfF ? 0.f : m_new));
        m = m_new;
        l *= alpha;
#pragma unroll
        for (int d = 0; d < ND; ++d) o[d] *= alpha;
      }
      const float m_use = m == kNegInfF ? 0.f : m;
#pragma unroll
      for (int kt = 0; kt < KT; ++kt)
#pragma unroll
        for (int i = 0; i < 16; ++i) {
          s[kt][i] = __builtin_amdgcn_exp2f(s[kt][i] - m_use);
          l += s[kt][i];
        }
    }
#pragma unroll
    for (int kt = 0; kt < KT; ++kt)
#pragma unroll
      for (int st = 0; st < 2; ++st) {
        u32x4 pw;
#pragma unroll
        for (int w = 0; w < 4; ++w) {
          const bf16x2 p = {(__bf16)s[kt][8 * st + 2 * w], (__bf16)s[kt][8 * st + 2 * w + 1]};
          pw[w] = __builtin_bit_cast(uint32_t, p);
        }
        const bf16x8 pb = __builtin_bit_cast(bf16x8, pw);
#pragma unroll
        for (int d = 0; d < ND; ++d) {
          // lane i of 16 names key i / 4 of four, elements 4 * (i % 4); it gets element i of all four
          const int row = 32 * kt + 16 * st + 4 * h + (lane & 15) / 4;
          const int e = 32 * d + 16 * ((lane >> 4) & 1) + 4 * (lane & 3);
          const i16x4 v0 = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_i16x4*)(sv + v_at<D>(row, e)));
          const i16x4 v1 = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_i16x4*)(sv + v_at<D>(row + 8, e)));
          typedef short i16x8 __attribute__((ext_vector_type(8)));
          const i16x8 va = __builtin_shufflevector(v0, v1, 0, 1, 2, 3, 4, 5, 6, 7);
          o[d] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, va), pb, o[d], 0, 0, 0);
        }
      }
  };

  // ---- the walk ---------------------------------------------------------------------------
  if (blk0 < blk1) {
    list_pages(page_base);
    load(blk0);
    store(blk0, 0);
    for (int blk = blk0; blk < blk1; ++blk) {
      const int buf = kBuffers == 2 ? (blk - blk0) & 1 : 0;
      const bool more = blk + 1 < blk1;
      if (more) load(blk + 1);
      // the block is in LDS, and nobody reads the other buffer any more
      if (kOwnKeys) wave_lds_sync();
      else lds_barrier();
      attend(blk, buf);
      if (kOwnKeys) wave_lds_sync();
      if (more) store(blk + 1, kBuffers == 2 ? buf ^ 1 : 0);
    }
  }
  l = sum_xor32(l);

  // ---- infinite and NaN values of edge blocks, to the rows that see them (the weight of a token that a
  // row sees is positive, so they are what they add up to)
  if constexpr (!kOwnKeys) {
    if (others) *s_others = 1;
    lds_barrier();
    others = *s_others != 0;
  }
  if (others) {
#pragma unroll 1
    for (int blk = max(blk0, lim_first / BN); blk < blk1; ++blk)
#pragma unroll 1
      for (int key = blk * BN + wk * BK; key < min(blk * BN + (wk + 1) * BK, lim_hi); ++key) {
        const int page = checked_page(table[key >> 4], a.n_pages, a.status);
        const uint8_t* v = a.v_cache + ((size_t)page * a.page_stride + (size_t)(g * 16 + key % 16) * D) * EB;
#pragma unroll
        for (int d = 0; d < ND; ++d)
#pragma unroll
          for (int i = 0; i < 16; ++i) {
            const int e = 32 * d + 8 * (i / 4) + 4 * h + i % 4;
            uint32_t bits;   // as fp32
            if constexpr (KV8) bits = (v[e] & 0x7f) == 0x7f ? 0x7fc00000u : 0u;
            else bits = (uint32_t)reinterpret_cast<const uint16_t*>(v)[e] << 16;
            if (key < lim && (bits & 0x7f800000u) == 0x7f800000u) o[d][i] += __uint_as_float(bits);
          }
      }
  }

  // ---- the result, or this split's part of it: outputs e .. e + 3 of the lane's row ----------
  const float v_scale = KV8 && a.v_scale ? a.v_scale[g] : 1.f;
  const size_t part = (size_t)split * a.runs.n_rows * Hq + out_row;
  auto emit = [&](const f32x4& x, int e) {
    if (n_valid > 1) *reinterpret_cast<f32x4*>(a.part_o + part * D + e) = x;
    else *reinterpret_cast<u32x2*>(a.out + out_row * D + e) = pack_outputs(x, v_scale, l);
  };
  auto emit_sums = [&]() {
    if (a.n_split > 1 && split == 0) a.part_n[out_row] = n_valid > 1 ? n_valid : 0;
    if (n_valid > 1) *reinterpret_cast<float2*>(a.part_ml + 2 * part) = make_float2(m, l);
  };

  if constexpr (WK == 1) {
    if (!real) return;
    if (h == 0) emit_sums();
#pragma unroll
    for (int d = 0; d < ND; ++d)
#pragma unroll
      for (int i = 0; i < 4; ++i)
        emit(f32x4{o[d][4 * i], o[d][4 * i + 1], o[d][4 * i + 2], o[d][4 * i + 3]}, 32 * d + 8 * i + 4 * h);
  } else {
    // Waves along the keys are joined through LDS, in their order: each takes a share of the
    // outputs (of every row) and reads it from all.
    static_assert(WR == 1 && 4 * ND % WK == 0, "whole shares");
    constexpr int kShare = 4 * ND / WK;           // groups of four outputs
    f32x4* so = reinterpret_cast<f32x4*>(s_kv);   // [WK][4 * ND][64]
    lds_barrier();
    s_ml[wk * 64 + lane] = make_float2(m, l);
#pragma unroll
    for (int f = 0; f < 4 * ND; ++f)
      so[(wk * 4 * ND + f) * 64 + lane] =
          f32x4{o[f / 4][4 * (f % 4)], o[f / 4][4 * (f % 4) + 1], o[f / 4][4 * (f % 4) + 2], o[f / 4][4 * (f % 4) + 3]};
    lds_barrier();
    if (!real) return;
    float f[WK];
    m = kNegInfF;
#pragma unroll
    for (int w = 0; w < WK; ++w) m = fmaxf(m, s_ml[w * 64 + lane].x);
    l = 0.f;
#pragma unroll
    for (int w = 0; w < WK; ++w) {
      const float2 ml = s_ml[w * 64 + lane];
      f[w] = __builtin_amdgcn_exp2f(ml.x - (m == kNegInfF ? 0.f : m));
      l += f[w] * ml.y;
    }
    if (wk == 0 && h == 0) emit_sums();
#pragma unroll
    for (int c = 0; c < kShare; ++c) {
      const int at = wk * kShare + c;
      f32x4 x = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int w = 0; w < WK; ++w) x += f[w] * so[(w * 4 * ND + at) * 64 + lane];
      emit(x, 8 * at + 4 * h);
    }
  }
}

// The tile of this workgroup: which sequence, which of its rows; false: there is none.
template <int ROWS>
__device__ __forceinline__ bool find_tile(const ExtendArgs& a, TileOf& t) {
  const int lane = threadIdx.x & 63, G = a.n_q_heads / a.n_kv_heads;
  int tile = blockIdx.y;
  // 256 sequences a round, four neighbours per lane
  constexpr int kPer = 4;
  for (int c = 0; c < a.runs.batch; c += 64 * kPer) {
    int at[kPer + 1], tiles[kPer], sum = 0;
#pragma unroll
    for (int i = 0; i <= kPer; ++i) at[i] = run_offset(a.runs, min(c + kPer * lane + i, a.runs.batch));
#pragma unroll
    for (int i = 0; i < kPer; ++i) {
      tiles[i] = (int)(((int64_t)max(0, at[i + 1] - at[i]) * G + ROWS - 1) / ROWS);
      sum += tiles[i];
    }
    const int incl = wave_incl_scan(sum);
    const uint64_t past = __ballot(incl > tile);
    if (past) {
      const int l = __builtin_ctzll(past);
      int left = tile - (__builtin_amdgcn_readlane(incl, l) - __builtin_amdgcn_readlane(sum, l));
      bool found = false;
#pragma unroll
      for (int i = 0; i < kPer; ++i) {
        const int n = __builtin_amdgcn_readlane(tiles[i], l);
        if (!found && left < n) {
          found = true;
          t.b = c + kPer * l + i;
          t.begin = __builtin_amdgcn_readlane(at[i], l);
          t.n_new = __builtin_amdgcn_readlane(at[i + 1], l) - t.begin;
          t.first = (n - 1 - left) * ROWS;   // the last rows see most keys: they start first
        }
        left -= found ? 0 : n;
      }
      t.n_rows = t.n_new * G;   // (n_rows * Hq < 2^31)
      t.s_b = max(0, min(a.runs.seq_lens[t.b], a.max_seq_len));
      return true;
    }
    tile -= __builtin_amdgcn_readlane(incl, 63);
  }
  return false;
}

// Tiles of 32 rows, four waves along the keys.
template <int D, bool KV8>
__global__ __launch_bounds__(256, 2) void extend_few_kernel(const ExtendArgs a) {
  __shared__ __attribute__((aligned(256))) uint16_t s_kv[kBodyLds<D, 1, 4, 1> / 2];
  __shared__ float2 s_ml[4 * 64];
  TileOf t;
  if (find_tile<32>(a, t)) extend_body<D, 1, 4, 1, KV8>(a, t, s_kv, s_ml, nullptr);
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
  if (t.n_rows - t.first <= 32) extend_body<D, 1, 8, 1, KV8>(a, t, s_kv, s_ml, nullptr);
  else extend_body<D, 8, 1, 2, KV8>(a, t, s_kv, s_ml, &s_others);
}

// Folds the splits' parts: D/4 lanes a (row, query head), four outputs each, splits in order.
template <int D>
__global__ __launch_bounds__(256) void extend_join_kernel(const ExtendArgs a, bool kv8) {
  constexpr int L = D / 4;
  const int64_t item = (int64_t)blockIdx.x * (256 / L) + threadIdx.x / L;
  const int e = 4 * (threadIdx.x % L);
  const int Hq = a.n_q_heads;
  const int first = a.runs.row_offsets ? run_offset(a.runs, 0) : 0;
  const int end = a.runs.row_offsets ? run_offset(a.runs, a.runs.batch) : a.runs.n_rows;
  const int row = (int)(item / Hq), head = (int)(item - (int64_t)row * Hq);
  if (row < first || row >= end) return;
  const size_t stride = (size_t)a.runs.n_rows * Hq;
  // 0: written by its only piece.  (Bounded: a run longer than the host's bound has rows without.)
  const int n = min(a.part_n[item], a.n_split);
  if (n <= 0) return;
  float m = kNegInfF, l = 0.f;
  f32x4 o = {0.f, 0.f, 0.f, 0.f};
  for (int s = 0; s < n; ++s) {
    const size_t part = s * stride + (size_t)item;
    const float2 ml = *reinterpret_cast<const float2*>(a.part_ml + 2 * part);
    const f32x4 x = *reinterpret_cast<const f32x4*>(a.part_o + part * D + e);
    const float m_new = fmaxf(m, ml.x), m_use = m_new == kNegInfF ? 0.f : m_new;
    const float f1 = __builtin_amdgcn_exp2f(m - m_use), f2 = __builtin_amdgcn_exp2f(ml.x - m_use);
    m = m_new;
    l = l * f1 + ml.y * f2;
    o = o * f1 + x * f2;
  }
  const float v_scale = kv8 && a.v_scale ? a.v_scale[head / (Hq / a.n_kv_heads)] : 1.f;
  *reinterpret_cast<u32x2*>(a.out + (size_t)item * D + e) = pack_outputs(o, v_scale, l);
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
