// Attention of runs of rows over the paged cache (Sec. 2, Eq. gqa_attention, for more than one query
// token of a sequence): what the kernels for causal runs and for trees of drafted tokens share.
//
// Mathematics.  A row is one (new token, query head) pair.  out = sum_t p_t v_t / sum_t p_t over the
// tokens t the row sees, p_t = 2^(s_t - m), s_t the scaled score in the log2 domain, m the running
// maximum: one pass over the keys, the sums rescaled when the maximum rises (Milakov and Gimelshein,
// "Online normalizer calculation for softmax", 2018).
//
// Work.  The rows of a run that share a KV head (token-major, the group's query heads next to each
// other) are cut into tiles; a workgroup takes a tile, and a piece of the keys that it sees.  A
// wave holds 32 rows and takes 32*KT keys of a block; WR waves stand along the rows, WK along the keys.
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
// a transposing read do): reads have no bank conflicts.  Storing blocks of e4m3 caches as bf16 or fp16 has: lanes store
// two 16-byte pieces of a row one after the other, 7.8e6 of the 3.05e7 LDS cycles of 12 trees over 10K-32K tokens.
//
// Precision.  Scores, maximum, sum and outputs are fp32.  The matrix cores take the inputs of the P V product in 16
// bits, so there a probability is rounded:
//   * causal runs, and trees in tiles of 256 rows of bf16 caches: to bf16, at most 2^-8 of each (see
//     tree_attn_kernel.hip for the price of a second term);
//   * trees in tiles of 32 rows of bf16 caches: to two bf16 terms, 2^-16 of each (kTwoTerms), which costs little
//     where the cache's bytes or a chain of loads decide;
//   * trees over e4m3 caches: to fp16, 2^-11 of each (kHalf).  fp16 holds every e4m3 value, and its conversions
//     and products are as fast as bf16's.
#pragma once

#include <algorithm>

#include "attend_lds.h"
#include "attn_tile.h"
#include "debug_check.h"
#include "runs.h"

namespace delta {
namespace {

typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef _Float16 f16x2 __attribute__((ext_vector_type(2)));
typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));
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

// What of a tile's keys a workgroup takes, and where its outputs go.
struct Piece {
  int g;              // KV head
  int blk0, blk1;     // blocks of keys (32 * KT * WK of them)
  bool whole;         // all that the tile sees: the result is written
  int note;           // what part_n gets for every row; -1: nothing.  (TREE: with the row's place in the tile from
                      // bit 20 on, except for 0)
  size_t part;        // the part: index of row 0 (TREE: of the tile; else of the call)
};

// The arguments of a kernel whose only parameter they are, read anew.  Kept from the kernel's start they take the
// scalar registers that the products' schedule needs (without them it waits for LDS before every product).
__device__ __forceinline__ ExtendArgs read_args() {
  typedef const __attribute__((address_space(4))) uint64_t* Kernarg;
  static_assert(sizeof(ExtendArgs) % 8 == 0, "whole words");
  struct Words {
    uint64_t w[sizeof(ExtendArgs) / 8];
  } words;
  Kernarg kernarg = (Kernarg)__builtin_amdgcn_kernarg_segment_ptr();
  asm volatile("" : "+s"(kernarg));
#pragma unroll
  for (size_t i = 0; i < sizeof(ExtendArgs) / 8; ++i) words.w[i] = kernarg[i];
  return __builtin_bit_cast(ExtendArgs, words);
}

// A value that is the same in all lanes, in a vector register.
__device__ __forceinline__ int held(int x) {
  asm volatile("" : "+v"(x));
  return x;
}

// Words of a row's mask at most, and tokens of a tile: their masks stand in LDS.
constexpr int kMostMaskWords = 16;
template <int ROWS>
constexpr int kMaskLds = (ROWS + 2) * kMostMaskWords;

// Loads 16 bytes a lane to LDS, lane after lane from byte `lds` on, past the registers.  Nothing but load_wait waits
// for it.
__device__ __forceinline__ void load_to_lds(const uint8_t* from, uint32_t lds) {
  uint32_t m0;   // (kept: the compiler takes it for its own)
  asm volatile("s_mov_b32 %0, m0\n\ts_mov_b32 m0, %1\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %2, off nt\n\ts_mov_b32 m0, %0"
               : "=&s"(m0)
               : "s"(lds), "v"(from)
               : "memory");
}
// All but the last N loads of the wave are done.  (Loads that the compiler knows of count too: then it waits longer.)
template <int N>
__device__ __forceinline__ void load_wait() {
  asm volatile("s_waitcnt vmcnt(%0)" ::"n"(N) : "memory");
}

// Two e4m3 values, in the lower or the upper half of a word, as fp16 or bf16.
template <bool HALF, bool HI>
__device__ __forceinline__ uint32_t e4m3x2_to(uint32_t w) {
  if (HALF) return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(w, 1.f, HI));
  return e4m3x2_to_bf16x2<HI>(w);
}

// What a row sees.  Causal runs: the tokens up to itself.  TREE: the tokens before the run, and of the
// run's rows those whose bits are set in the row's mask.
//
// RING: the blocks are brought by loads that go to LDS, kRing - 1 of them under way while one is worked on; bf16
// blocks where the products read them, e4m3 ones to LDS of the wave that loads them, which makes bf16 of them
// (the two buffers of the other forms) one block ahead.
template <int D, int WR, int WK, int KT, bool KV8, bool TREE, bool RING = false>
__device__ __forceinline__ void extend_body(const ExtendArgs& a, const TileOf& t, const Piece& piece,
                                            uint16_t* s_kv, float2* s_ml, int* s_others, int* s_pages = nullptr,
                                            uint32_t* s_masks = nullptr) {
  static_assert(!RING || WR > 1, "waves that share blocks");
  constexpr int NW = WR * WK, T = 64 * NW;
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
  int tid = threadIdx.x;
  // (a workgroup takes several tiles: what follows from the lane is formed for each anew, as kept in registers
  // from tile to tile it would not fit them)
  if (TREE) asm volatile("" : "+v"(tid));
  const int lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int wr = wave % WR, wk = wave / WR;
  const int n = lane & 31, h = lane >> 5;
  const int g = piece.g;
  const int Hq = a.n_q_heads, G = Hq / a.n_kv_heads;

  // Waves that share no rows share no keys either: each brings its own keys to its own LDS, without
  // barriers, and needs one buffer of it.
  constexpr bool kOwnKeys = WR == 1;
  constexpr int kBuffers = kOwnKeys ? 1 : 2;
  // the inputs of the P V product (see Precision)
  constexpr bool kHalf = TREE && KV8, kTwoTerms = TREE && !KV8 && WR == 1;
  // (fp16 probabilities stand for 2^15 times as much, in the sums as well, so that those from 2^-29 on are normal)
  constexpr float kLift = kHalf ? 15.f : 0.f;
  auto add_values = [&](const bf16x8& v, const u32x4& p, const f32x16& c) {
    if constexpr (kHalf)
      return __builtin_amdgcn_mfma_f32_32x32x16_f16(__builtin_bit_cast(f16x8, v), __builtin_bit_cast(f16x8, p), c, 0, 0, 0);
    else
      return __builtin_amdgcn_mfma_f32_32x32x16_bf16(v, __builtin_bit_cast(bf16x8, p), c, 0, 0, 0);
  };
  constexpr int kBlock = BN * D;        // elements of a K or V block
  const int b = t.b, n_new = t.n_new, s_b = t.s_b, n_tile_rows = t.n_rows, begin = t.begin;
  // this lane's row: token j of the run, query head g * G + head
  const int r0 = t.first + 32 * wr;
  const int r = min(r0 + n, n_tile_rows - 1);
  const bool real = r0 + n < n_tile_rows;
  const bool active = r0 < n_tile_rows;                               // some row of the wave is
  const int j = r / G, head = g * G + (r - j * G);
  const size_t out_row = (size_t)(begin + j) * Hq + head;
  const int base = s_b - n_new;                                       // token index of the run's row 0
  const int lim = TREE ? s_b : max(0, base + j + 1);                  // keys from here on the row does not see
  auto lim_of = [&](int row) { return max(0, base + min(row, n_tile_rows - 1) / G + 1); };
  // of the wave's rows: keys that all see, and that none sees
  const int lim_lo = TREE ? max(0, base) : lim_of(r0), lim_hi = TREE ? s_b : lim_of(r0 + 31);
  // TREE: which of keys key0 .. key0 + 31 the row sees (bit 0: key0), from the masks of the tile's tokens in LDS
  const int words = TREE ? min(kMostMaskWords, min(a.mask_words, (n_new + 31) / 32)) : 0;
  const int j0 = t.first / G;
  auto mask_word = [&](int w) -> uint32_t {
    return w < 0 ? ~0u /* tokens before the run */ : w >= words ? 0u : s_masks[(j - j0) * words + w];
  };
  auto seen_of = [&](int key0) -> uint32_t {
    const int w = (key0 - base) >> 5, shift = (key0 - base) & 31;
    return __builtin_amdgcn_alignbit(mask_word(w + 1), mask_word(w), shift);
  };

  const int blk0 = piece.blk0, blk1 = piece.blk1;

  const float scale = KV8 && a.k_scale ? a.scale_log2 * a.k_scale[g] : a.scale_log2;
  bf16x8 q[NK];
#pragma unroll
  for (int ks = 0; ks < NK; ++ks)
    q[ks] = __builtin_bit_cast(bf16x8, *reinterpret_cast<const u32x4*>(a.q + out_row * D + 16 * ks + 8 * h));
  // what else of the tile is looked up, its loads together: the first pages, and masks
  const int32_t* table = a.runs.page_table + (size_t)b * a.runs.max_pages;
  const int last_page = max(0, (s_b - 1) >> 4);
  int base_page = blk0 * (BN / 16);
  if constexpr (TREE) {
    const int n_words = ((min(t.first + 32 * WR, n_tile_rows) - 1) / G - j0 + 1) * words;
    auto mask_at = [&](int i) {
      const int row = i / words, w = i - row * words, left = n_new - 32 * w;
      return a.masks[(size_t)(begin + j0 + row) * a.mask_words + w] & (left >= 32 ? ~0u : (1u << left) - 1u);
    };
    auto page_at = [&](int i) { return base_page + i <= last_page ? table[base_page + i] : 0; };
    const int page = RING && blk0 < blk1 ? page_at(tid) : 0;
    const uint32_t mask = tid < n_words ? mask_at(tid) : 0u;
    if (tid < n_words) s_masks[tid] = mask;
    for (int i = tid + T; i < n_words; i += T) s_masks[i] = mask_at(i);
    if (RING && blk0 < blk1) {
      s_pages[tid] = checked_page(page, a.n_pages, a.status);
      for (int i = tid + T; i < kRingPages; i += T)
        if (base_page + i <= last_page) s_pages[i] = checked_page(page_at(i), a.n_pages, a.status);
    }
    if (kOwnKeys || RING) lds_barrier();   // (the others have one before the first block)
  }
  // they are waited for here: a wait for their first use, inside the loop, would also wait for the
  // loads of the next block in every round
#pragma unroll
  for (int ks = 0; ks < NK; ++ks) asm volatile("" : "+v"(q[ks]));

  float m = kNegInfF, l = 0.f;
  f32x16 o[ND];
#pragma unroll
  for (int i = 0; i < ND; ++i) o[i] = f32x16{};

  // ---- blocks: pages of the next 64 (one per lane), loads, LDS ------------------------------
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
  const int lim_first = TREE ? lim_lo : lim_of(t.first);
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
            wv[2 * w] = e4m3x2_to<kHalf, false>(vr[i][2 * half + w]);
            wv[2 * w + 1] = e4m3x2_to<kHalf, true>(vr[i][2 * half + w]);
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
    auto key_part = [&](int kt, int ks) {
      return __builtin_bit_cast(bf16x8, *reinterpret_cast<const u32x4*>(sk + k_at<D>(32 * kt + n, 2 * ks + h)));
    };
    auto value_part = [&](int step, int d) {   // of 16 keys
      // lane i of 16 names key i / 4 of four, elements 4 * (i % 4); it gets element i of all four
      const int row = 16 * step + 4 * h + (lane & 15) / 4;
      const int e = 32 * d + 16 * ((lane >> 4) & 1) + 4 * (lane & 3);
      const i16x4 v0 = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_i16x4*)(sv + v_at<D>(row, e)));
      const i16x4 v1 = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_i16x4*)(sv + v_at<D>(row + 8, e)));
      typedef short i16x8 __attribute__((ext_vector_type(8)));
      const i16x8 va = __builtin_shufflevector(v0, v1, 0, 1, 2, 3, 4, 5, 6, 7);
      return __builtin_bit_cast(bf16x8, va);
    };
    // kGrouped: the reads of a row of products stand together before it (`read`: they are made by there).  Left to the
    // compiler, whether each product waits for a read of its own depends on how many scalar registers are left.
    constexpr bool kGrouped = TREE && WR > 1;
    auto read = [](bf16x8& x) { asm volatile("" : "+v"(x)); };
    bf16x8 v_part[2][ND];
#pragma unroll
    for (int kt = 0; kt < KT; ++kt) {
      s[kt] = f32x16{};
      if constexpr (kGrouped) {
        bf16x8 k_part[NK];
#pragma unroll
        for (int ks = 0; ks < NK; ++ks) k_part[ks] = key_part(kt, ks);
#pragma unroll
        for (int ks = 0; ks < NK; ++ks) read(k_part[ks]);
#pragma unroll
        for (int ks = 0; ks < NK; ++ks)
          s[kt] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(k_part[ks], q[ks], s[kt], 0, 0, 0);
      } else {
#pragma unroll
        for (int ks = 0; ks < NK; ++ks)
          s[kt] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(key_part(kt, ks), q[ks], s[kt], 0, 0, 0);
      }
    }
    if constexpr (kGrouped) {
#pragma unroll
      for (int st = 0; st < 2; ++st)
#pragma unroll
        for (int d = 0; d < ND; ++d) v_part[st][d] = value_part(st, d);
    }
    {
// a scaled score is rounded before the maximum and the difference see it: contracted into the
// difference's fma, the maximum's own rounding error would be left in the exponent
#pragma clang fp contract(off)
#pragma unroll
      for (int kt = 0; kt < KT; ++kt) s[kt] *= scale;
      if (key0 + BK > lim_lo) {   // some row of the wave does not see all of these keys
#pragma unroll
        for (int kt = 0; kt < KT; ++kt) {
          const uint32_t seen = TREE ? seen_of(key0 + 32 * kt) >> (4 * h) : 0u;
#pragma unroll
          for (int i = 0; i < 16; ++i) {
            const int key = key0 + 32 * kt + 8 * (i / 4) + 4 * h + i % 4;
            const bool sees = TREE ? (seen >> (8 * (i / 4) + i % 4)) & 1u : key < lim;
            s[kt][i] = sees ? s[kt][i] : kNegInfF;
          }
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
      const float m_use = (m == kNegInfF ? 0.f : m) - kLift;
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
        u32x4 pw, rest;
#pragma unroll
        for (int w = 0; w < 4; ++w) {
          const float p0 = s[kt][8 * st + 2 * w], p1 = s[kt][8 * st + 2 * w + 1];
          if constexpr (kHalf) {
            pw[w] = __builtin_bit_cast(uint32_t, f16x2{(_Float16)p0, (_Float16)p1});
          } else {
            pw[w] = __builtin_bit_cast(uint32_t, bf16x2{(__bf16)p0, (__bf16)p1});
            if constexpr (kTwoTerms)
              rest[w] = __builtin_bit_cast(uint32_t, bf16x2{(__bf16)(p0 - __uint_as_float(pw[w] << 16)),
                                                            (__bf16)(p1 - __uint_as_float(pw[w] & 0xffff0000u))});
          }
        }
        if constexpr (kGrouped) {
#pragma unroll
          for (int d = 0; d < ND; ++d) read(v_part[st][d]);
#pragma unroll
          for (int d = 0; d < ND; ++d) {
            o[d] = add_values(v_part[st][d], pw, o[d]);
            if (kt + 1 < KT) v_part[st][d] = value_part(2 * (kt + 1) + st, d);
          }
        } else {
          bf16x8 v[ND];
#pragma unroll
          for (int d = 0; d < ND; ++d) o[d] = add_values(v[d] = value_part(2 * kt + st, d), pw, o[d]);
          if constexpr (kTwoTerms) {
#pragma unroll
            for (int d = 0; d < ND; ++d) o[d] = add_values(v[d], rest, o[d]);
          }
        }
      }
  };

  // ---- the walk ---------------------------------------------------------------------------
  if constexpr (RING) {
    const uint32_t s_kv_at = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) uint16_t*)s_kv;
    constexpr int kLoads = 2 * NL;                           // of a wave and block
    typedef RawRing<D, NW, BN> Raw;                          // e4m3: the waves' own LDS
    // a lane's 16 bytes of the rows of a load; bf16: that which stands in its place of the permuted rows (the
    // rows of a wave's loads lie a multiple of 16 apart, or of what else the permutation knows of a row)
    const int lr = lane / CPR, lc = lane % CPR;
    const int row0 = wave * RPW + lr;
    static_assert(KV8 || NW * RPW % 16 == 0, "one permutation for all loads of a wave");
    const uint32_t k_lane = KV8 ? lane16 : (uint32_t)(lr * D * 2 + 2 * (k_at<D>(row0, lc) - row0 * D));
    const uint32_t v_lane = KV8 ? lane16 : (uint32_t)(lr * D * 2 + 2 * (v_at<D>(row0, 8 * lc) - row0 * D));
    auto list = [&](int first) {   // the next pages, of the blocks from `first` on
      lds_barrier();
      base_page = first * (BN / 16);
      for (int i = tid; i < kRingPages; i += T)
        if (base_page + i <= last_page) s_pages[i] = checked_page(table[base_page + i], a.n_pages, a.status);
      lds_barrier();
    };
    auto issue = [&](int blk) {
      if ((blk + 1) * (BN / 16) > base_page + kRingPages) list(blk);
      const int stage = (blk - blk0) % kRing;
#pragma unroll
      for (int i = 0; i < NL; ++i) {
        const int row = row_of(i);
        if (kPieces % T && row >= BN) break;
        // (blocks end past the last page: it is loaded in place of those that are not)
        // (in vector registers: scalar ones are short)
        const uint32_t page = s_pages[min(blk * (BN / 16) + row / 16, last_page) - base_page];
        const size_t at = ((size_t)page * (uint32_t)a.page_stride + (uint32_t)((g * 16 + row % 16) * D)) * EB;
        const uint32_t to = s_kv_at + (KV8 ? Raw::at(wave, stage, i)
                                           : (stage * 2 * kBlock + row * D) * 2);
        load_to_lds(a.k_cache + at + k_lane, to);
        load_to_lds(a.v_cache + at + v_lane, to + (KV8 ? 1024 : kBlock * 2));
      }
    };
    // waits until the loads of a block are done after which `after` more were issued
    auto arrived = [&](int after) {
      static_assert(kRing == 4, "cases below");
      if (after >= 3) load_wait<3 * kLoads>();
      else if (after == 2) load_wait<2 * kLoads>();
      else if (after == 1) load_wait<kLoads>();
      else load_wait<0>();
    };
    if (blk0 < blk1) {
      if constexpr (KV8) {
        auto convert = [&](int blk) {
          arrived(min(kRing - 1, blk1 - 1 - blk));
          const int stage = (blk - blk0) % kRing;
#pragma unroll
          for (int i = 0; i < NL; ++i) {
            if (kPieces % T && !Raw::has(wave, i)) break;
            const uint8_t* raw = reinterpret_cast<const uint8_t*>(s_kv) + Raw::at(wave, stage, i) + lane16;
            kr[i] = *reinterpret_cast<const u32x4*>(raw);
            vr[i] = *reinterpret_cast<const u32x4*>(raw + 1024);
          }
          store(blk, (blk - blk0) & 1);
          wave_lds_sync();   // (its own LDS has been read)
          if (blk + kRing < blk1) issue(blk + kRing);
        };
        for (int i = 0; i < kRing; ++i)
          if (blk0 + i < blk1) issue(blk0 + i);
        convert(blk0);
        for (int blk = blk0; blk < blk1; ++blk) {
          lds_barrier();   // the block is in LDS, and nobody reads the other buffer any more
          if (blk + 1 < blk1) convert(blk + 1);
          attend(blk, (blk - blk0) & 1);
        }
      } else {
        for (int i = 0; i < kRing - 1; ++i)
          if (blk0 + i < blk1) issue(blk0 + i);
        for (int blk = blk0; blk < blk1; ++blk) {
          const int stage = (blk - blk0) % kRing;
          arrived(min(kRing - 2, blk1 - 1 - blk));
          lds_barrier();   // all waves' loads of the block are done, and nobody reads the block before it any more
          if (blk + kRing - 1 < blk1) issue(blk + kRing - 1);
          if ((blk + 1) * BN > lim_first) {   // infinite and NaN values, see store
            uint32_t seen = 0;
            u32x4* sv = reinterpret_cast<u32x4*>(s_kv + stage * 2 * kBlock + kBlock);
            u32x4 x[NL];
#pragma unroll
            for (int i = 0; i < NL; ++i) {
              const int at = i * T + tid;
              if (kPieces % T && at >= kPieces) break;
              x[i] = sv[at];
              if (blk * BN + at / CPR >= s_b) x[i] = u32x4{0u, 0u, 0u, 0u};
#pragma unroll
              for (int w = 0; w < 4; ++w) look_for_others<KV8>(x[i][w], seen);
            }
            const bool some = __any(has_others<KV8>(seen));
            others |= some;
            if (some || (blk + 1) * BN > s_b) {
#pragma unroll
              for (int i = 0; i < NL; ++i) {
                const int at = i * T + tid;
                if (kPieces % T && at >= kPieces) break;
#pragma unroll
                for (int w = 0; w < 4; ++w) x[i][w] = without_others<KV8>(x[i][w]);
                sv[at] = x[i];
              }
            }
            lds_barrier();
          }
          attend(blk, stage);
        }
      }
    }
  } else if (blk0 < blk1) {
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
    const ExtendArgs z = TREE ? read_args() : a;
    const int32_t* table = z.runs.page_table + (size_t)b * z.runs.max_pages;
#pragma unroll 1
    for (int blk = max(blk0, lim_first / BN); blk < blk1; ++blk)
#pragma unroll 1
      for (int key = blk * BN + wk * BK; key < min(blk * BN + (wk + 1) * BK, lim_hi); ++key) {
        const int page = checked_page(table[key >> 4], z.n_pages, z.status);
        const bool sees = TREE ? seen_of(key) & 1u : key < lim;
        const uint8_t* v = z.v_cache + ((size_t)page * z.page_stride + (size_t)(g * 16 + key % 16) * D) * EB;
#pragma unroll
        for (int d = 0; d < ND; ++d)
#pragma unroll
          for (int i = 0; i < 16; ++i) {
            const int e = 32 * d + 8 * (i / 4) + 4 * h + i % 4;
            uint32_t bits;   // as fp32
            if constexpr (KV8) bits = (v[e] & 0x7f) == 0x7f ? 0x7fc00000u : 0u;
            else bits = (uint32_t)reinterpret_cast<const uint16_t*>(v)[e] << 16;
            if (sees && (bits & 0x7f800000u) == 0x7f800000u) o[d][i] += __uint_as_float(bits);
          }
      }
  }

  // ---- the result, or this split's part of it: outputs e .. e + 3 of the lane's row ----------
  const ExtendArgs z = TREE ? read_args() : a;
  const float v_scale = KV8 && z.v_scale ? z.v_scale[g] : 1.f;
  const size_t part = piece.part + (TREE ? 32 * wr + n : out_row);
  f32x4* part_o = reinterpret_cast<f32x4*>(z.part_o + part * D);
  u32x2* out = reinterpret_cast<u32x2*>(z.out + out_row * D);
  auto emit = [&](const f32x4& x, int e) {
    if (!piece.whole) part_o[e / 4] = x;
    else out[e / 4] = pack_outputs(x, v_scale, l);
  };
  auto emit_sums = [&]() {
    if (piece.note >= 0) z.part_n[out_row] = TREE && piece.note ? piece.note | (32 * wr + n) << 20 : piece.note;
    if (!piece.whole) *reinterpret_cast<float2*>(z.part_ml + 2 * part) = make_float2(m, l);
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
    static_assert(4 * ND % WK == 0, "whole shares");
    constexpr int kShare = 4 * ND / WK;           // groups of four outputs
    f32x4* so = reinterpret_cast<f32x4*>(s_kv) + wr * WK * 4 * ND * 64;   // [WK][4 * ND][64] of the rows
    s_ml += wr * WK * 64;
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

// The piece that split blockIdx.z of KV head blockIdx.x takes of a causal tile of BM rows, in blocks of BN keys;
// false: none.
template <int BM, int BN>
__device__ __forceinline__ bool causal_piece(const ExtendArgs& a, const TileOf& t, Piece& p) {
  const int G = a.n_q_heads / a.n_kv_heads, split = blockIdx.z;
  const int last = min(t.first + BM - 1, t.n_rows - 1) / G;
  const int n_blocks = (max(0, t.s_b - t.n_new + last + 1) + BN - 1) / BN;
  // pieces of one length whatever the sequence's: a short sequence has fewer
  const int per_split = a.split_keys / BN;
  const int n_valid = max(1, (n_blocks + per_split - 1) / per_split);
  if (split >= n_valid) return false;
  p.g = blockIdx.x;
  p.blk0 = split * per_split;
  p.blk1 = min(n_blocks, p.blk0 + per_split);
  p.whole = n_valid == 1;
  p.note = a.n_split > 1 && split == 0 ? (n_valid > 1 ? n_valid : 0) : -1;
  p.part = (size_t)split * a.runs.n_rows * a.n_q_heads;
  return true;
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

}  // namespace
}  // namespace delta
