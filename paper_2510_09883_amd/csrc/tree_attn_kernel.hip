// Attention of trees of drafted tokens over the paged cache: every row of a run sees the tokens before
// the run and the rows of the run that its mask names.
//
// The mathematics, the tile step and the LDS layouts are attend_runs.h's; a row's mask is looked at only in
// the blocks that hold rows of the run.
//
// Work.  Rows of a run that share a KV head form tiles of up to 256 (32, where no run is longer), and all tiles see
// the whole sequence.  Sequences differ in length and a batch has few of them, so up to 256 sequences are shared
// out evenly: groups of workgroups, one for each KV head (which then walk the same pages at the same time), take equal
// shares of the tiles' blocks of keys, found from the lengths on the device (make_cut).  A tile whose blocks fall
// to several groups leaves parts (two at most per workgroup: its first and its last tile), which a second
// launch joins.
//   * tiles of 256 rows: eight waves, one workgroup a CU.  Up to 128 rows the waves stand 4 x 2 (along the rows x along
//     the keys), above 8 x 1.  Blocks come through a ring in LDS (attend_runs.h); only e4m3 blocks of up to 128 rows
//     wait in registers and are twice as long, which leaves the waves more products between two barriers (32/8 heads,
//     16 sequences of 4K-16K, 32 rows each: 151 us, through the ring 163; bf16 by registers 183, through the ring 175).
//   * tiles of 32 rows (no longer run, or little to walk): four waves along the keys, each with keys of its own.
//
// Precision.  A probability meets the values in 16 bits (attend_runs.h).  Two bf16 terms for each, what the first leaves
// as well, cost tiles of 32 rows little, us without and with them: 16 sequences of 4K-16K tokens, 8 nodes, 32/8 heads 131
// and 132, 32 short ones 10.1 and 9.9, one tree of 16 behind 8192 tokens, 28/4 heads, 19.8 and 20.5, one of 64 behind 2048
// 20.3 and 21.5.  Tiles of 256 rows would pay for them (16 sequences of 4K-16K, 32/8 heads, 16 nodes 147 and 169, 32
// nodes 178 and 209, 64 of each 238 and 300) and keep the one: 1.69e-3 rms off float64 instead of the output's own
// rounding's 1.66e-3.  e4m3 caches: two bf16 terms took 284 where one takes 167 (12 trees of 8 to 24 nodes, 40/8 heads),
// fp16 169.
//
// Bound (medians of 200 dispatches).  256 rows: issue, at the lower clock that loads and products together leave: 16
// trees of 64 nodes behind 4K-16K tokens, 32/8 heads, 237 us (763 TFLOP/s; the least 217, 835) at 2.01 GHz, VALU 50 %
// and MFMA 39 % of the SIMDs' cycles, and 12 for the join, which reads 48 MB of parts.  In an earlier state, 232 us
// together, taking the loads out left 164, taking the products out 154.
// 33 to 128 rows of bf16: HBM, 16 of 4K-16K with 16 nodes 128 us and 5 (in a graph 147 together, 4.7 TB/s); of e4m3:
// phases that follow one another between the barriers (loads, conversion, products, softmax; VALU 38 %, LDS 32 %, MFMA
// 26 %), 12 of 10K-32K with 8 to 24 nodes, 40/8 heads, 169 us and 7.  Measured slower or equal there: tiles of 128 rows by
// four waves, two workgroups a CU (bf16 -9 % to +3 %, e4m3 +18 % to +26 %), e4m3 blocks through a ring of two (+1 % to
// +4 %).
// Few rows: 16 of 4K-16K with 8 nodes 117 us and 5 (in a graph 132 together, 5.4 TB/s; e4m3 76 and 5); with a row of
// units per head instead of groups that walk the same pages at the same time 5 % more.  One tree of 16 behind 8192
// tokens, 28/4 heads: 17.7 and 4.0 for the join; behind 64 tokens, in one launch, 7.4 in a graph: the chain offsets ->
// queries, masks and pages -> blocks.
#include "attend_runs.h"
#include "drafts.h"

namespace delta {
namespace {

// Keys of a block and its units for tiles of so many rows: what a CU takes for it while all are busy, in about 0.14 us.
struct Form {
  int keys, units;
};
template <bool WIDE, bool KV8>
__device__ __forceinline__ Form form_of(int rows) {
  if (!WIDE) return Form{128, KV8 ? 4 : 8};
  if (rows <= 128) return KV8 ? Form{128, 6} : Form{64, 4};
  return Form{64, 6};
}

// The sequences of a shared call, in LDS.
struct Cut {
  int start[kCutBatch + 1];   // units (PIECES: pieces) before sequence b
  int begin[kCutBatch + 1];   // first row of its run
  int len[kCutBatch];         // its tokens
  int chunk;                  // units of a workgroup's part
};

struct TileUnits {
  Form form;
  int blocks, units;          // units: of the blocks alone
};
template <bool WIDE, bool KV8>
__device__ __forceinline__ TileUnits units_of(int rows, int len) {
  TileUnits u;
  u.form = form_of<WIDE, KV8>(rows);
  u.blocks = max(1, (len + u.form.keys - 1) / u.form.keys);
  u.units = u.blocks * u.form.units;
  return u;
}
// Blocks of a piece of so many units (rounded up, so that there are no more pieces than workgroups), and the pieces of a tile.
__device__ __forceinline__ int blocks_of(const TileUnits& u, int chunk) {
  return (chunk + u.form.units - 1) / u.form.units;
}
__device__ __forceinline__ int pieces_of(const TileUnits& u, int chunk) {
  const int per = blocks_of(u, chunk);
  return (u.blocks + per - 1) / per;
}

// Fills the cut: four sequences a lane of the first wave.
//
// The tiles' units stand in one row, kTileUnits for each and its blocks', and a workgroup takes an equal part of it, a
// tile's end and the next one's beginning too.  PIECES: every tile is cut into pieces of a length that makes no more of
// them than there are workgroups, and a workgroup takes one.
template <bool WIDE, bool KV8, bool PIECES>
__device__ __forceinline__ void make_cut(const ExtendArgs& a, Cut& cut) {
  constexpr int ROWS = WIDE ? 256 : 32, kPer = kCutBatch / 64;
  if (threadIdx.x < 64) {
    const int lane = threadIdx.x, G = a.n_q_heads / a.n_kv_heads, B = a.runs.batch,
              W = gridDim.x / a.n_kv_heads;   // groups
    int at[kPer + 1], len[kPer], full[kPer], rest[kPer];
#pragma unroll
    for (int i = 0; i <= kPer; ++i) at[i] = run_offset(a.runs, min(kPer * lane + i, B));
#pragma unroll
    for (int i = 0; i < kPer; ++i) len[i] = max(0, min(a.runs.seq_lens[min(kPer * lane + i, B - 1)], a.max_seq_len));
    int tiles = 0, units = 0;
#pragma unroll
    for (int i = 0; i < kPer; ++i) {
      const int rows = max(0, at[i + 1] - at[i]) * G;
      full[i] = rows / ROWS, rest[i] = rows % ROWS;
      tiles += full[i] + (rest[i] > 0);
      units += full[i] * units_of<WIDE, KV8>(ROWS, len[i]).units + (rest[i] ? units_of<WIDE, KV8>(rest[i], len[i]).units : 0);
    }
    tiles = __builtin_amdgcn_readlane(wave_incl_scan(tiles), 63);
    const int total = __builtin_amdgcn_readlane(wave_incl_scan(units), 63);
    // (with pieces there are fewer tiles than workgroups: every tile's last piece may be short)
    const int chunk = max(kLeastUnits, PIECES ? (total + max(1, W - tiles) - 1) / max(1, W - tiles)
                                              : (total + kTileUnits * tiles + W - 1) / W);
    int sum = 0, own[kPer];
#pragma unroll
    for (int i = 0; i < kPer; ++i) {
      const TileUnits f = units_of<WIDE, KV8>(ROWS, len[i]), r = units_of<WIDE, KV8>(rest[i], len[i]);
      own[i] = PIECES ? full[i] * pieces_of(f, chunk) + (rest[i] ? pieces_of(r, chunk) : 0)
                      : full[i] * (kTileUnits + f.units) + (rest[i] ? kTileUnits + r.units : 0);
      sum += own[i];
    }
    int before = wave_incl_scan(sum) - sum;
#pragma unroll
    for (int i = 0; i < kPer; ++i) {
      cut.start[kPer * lane + i] = before;
      cut.begin[kPer * lane + i] = at[i];
      cut.len[kPer * lane + i] = len[i];
      before += own[i];
    }
    if (lane == 63) {
      cut.start[kCutBatch] = before;
      cut.begin[kCutBatch] = at[kPer];
      cut.chunk = chunk;
    }
  }
  __syncthreads();
}

// LDS of a workgroup.
template <int D, bool WIDE, bool KV8>
constexpr int kTreeLds = WIDE ? std::max(KV8 ? kBodyLds<D, 4, 2, 2> : kBodyLds<D, 4, 2, 1, true, false>, kBodyLds<D, 8, 1, 2, true, KV8>)
                              : kBodyLds<D, 1, 4, 1>;

template <int D, bool WIDE, bool KV8>
__device__ __forceinline__ void attend_tile(const ExtendArgs& a, const TileOf& t, const Piece& p, uint16_t* s_kv,
                                            float2* s_ml, int* s_others, int* s_pages, uint32_t* s_masks) {
  if constexpr (!WIDE) {
    extend_body<D, 1, 4, 1, KV8, true>(a, t, p, s_kv, s_ml, nullptr, nullptr, s_masks);
  } else {
    const int rows = t.n_rows - t.first;
    if (rows > 128) extend_body<D, 8, 1, 2, KV8, true, true>(a, t, p, s_kv, s_ml, s_others, s_pages, s_masks);
    else if constexpr (KV8) extend_body<D, 4, 2, 2, true, true>(a, t, p, s_kv, s_ml, s_others, nullptr, s_masks);
    else extend_body<D, 4, 2, 1, false, true, true>(a, t, p, s_kv, s_ml, s_others, s_pages, s_masks);
  }
}

template <int D, bool WIDE, bool KV8, bool PIECES>
__global__ __launch_bounds__(WIDE ? 512 : 256, WIDE ? 1 : 2) void tree_attn_kernel(const ExtendArgs args) {
  constexpr int ROWS = WIDE ? 256 : 32;
  __shared__ __attribute__((aligned(256))) uint16_t s_kv[kTreeLds<D, WIDE, KV8> / 2];
  __shared__ float2 s_ml[(WIDE ? 8 : 4) * 64];
  __shared__ int s_pages[WIDE ? kRingPages : 1];
  __shared__ uint32_t s_masks[kMaskLds<WIDE ? 256 : 32>];
  __shared__ int s_others;   // some wave has met infinite or NaN values in an edge block
  __shared__ Cut cut;
  make_cut<WIDE, KV8, PIECES>(args, cut);
  const int G = args.n_q_heads / args.n_kv_heads, lane = threadIdx.x & 63;
  // (what is read of LDS is the same in all lanes; the compiler is told so)
  auto uniform = [](int x) { return __builtin_amdgcn_readfirstlane(x); };
  const int total = uniform(cut.start[kCutBatch]);
  int chunk = uniform(cut.chunk);
  const int part = PIECES ? 1 : chunk;   // of the row, a group's
  const int group = blockIdx.x / args.n_kv_heads;
  if ((int64_t)group * part >= total) return;
  int pos = group * part;
  int end = min(total, pos + part);
  int b = 0;   // the sequence of pos
#pragma unroll
  for (int i = 0; i < kCutBatch / 64; ++i) b += __popcll(__ballot(cut.start[64 * i + lane + 1] <= pos));

#pragma clang loop unroll(disable)
  while (pos < end) {
    const ExtendArgs a = read_args();
    while (b < kCutBatch - 1 && pos >= uniform(cut.start[b + 1])) ++b;
    TileOf t;
    t.b = b;
    t.begin = uniform(cut.begin[b]);
    t.n_new = uniform(cut.begin[b + 1]) - t.begin;
    t.n_rows = t.n_new * G;
    t.s_b = uniform(cut.len[b]);
    const int full = t.n_rows / ROWS;
    int at = pos - uniform(cut.start[b]);  // into the sequence's part of the row
    TileUnits u = units_of<WIDE, KV8>(ROWS, t.s_b);
    auto length_of = [&](const TileUnits& x) { return PIECES ? pieces_of(x, chunk) : kTileUnits + x.units; };
    int length = length_of(u), tile;
    if (at >= full * length) {             // the last, partial tile
      at -= full * length;
      tile = full;
      u = units_of<WIDE, KV8>(t.n_rows - full * ROWS, t.s_b);
      length = length_of(u);
    } else {
      tile = at / length;
      at -= tile * length;                 // into the tile
    }
    t.first = tile * ROWS;
    const int start = pos - at, group = blockIdx.x / a.n_kv_heads;
    Piece p;
    p.g = blockIdx.x - group * a.n_kv_heads;
    int group_last;                        // the group that has the tile's last block
    if constexpr (PIECES) {
      const int per = blocks_of(u, chunk);
      p.blk0 = at * per;
      p.blk1 = min(u.blocks, p.blk0 + per);
      group_last = group + length - 1;
    } else {
      // block i is the group's that has unit kTileUnits + i * form.units
      auto block_from = [&](int unit) {
        return min(u.blocks, (max(0, unit - kTileUnits) + u.form.units - 1) / u.form.units);
      };
      p.blk0 = block_from(at);
      p.blk1 = block_from(end - start);
      group_last = (start + kTileUnits + (u.blocks - 1) * u.form.units) / chunk;
      pos = min(end, start + length);
    }
    if (!PIECES && p.blk0 >= p.blk1) continue;
    const bool first = p.blk0 == 0, last = p.blk1 == u.blocks;
    p.whole = first && last;
    // where a tile's parts are: the first in its workgroup's second place, the others in the first places of the next
    // groups' workgroups
    p.part = (size_t)(2 * blockIdx.x + first) * ROWS;
    p.note = first ? (last ? 0 : (group_last - group + 1) | group << 10) : -1;
    if (t.s_b == 0) p.blk1 = 0;            // (no keys: its one block, which is the workgroup's, is none)
    lds_barrier();                         // (the tile before has read its LDS)
    if (threadIdx.x == 0) s_others = 0;    // (the walk's first barrier is before any use)
    // (what the compiler does not see to be the same in all lanes would cost registers that the tile has not)
    t.b = uniform(t.b), t.first = uniform(t.first), t.n_rows = uniform(t.n_rows);
    p.g = uniform(p.g), p.blk0 = uniform(p.blk0), p.blk1 = uniform(p.blk1);
    // (and what is not needed before the tile is done waits in vector registers, of which there are enough)
    p.note = held(p.note), p.whole = held(p.whole), p.part = (uint32_t)held((int)p.part);
    const int pos_held = held(pos), end_held = held(end), chunk_held = held(chunk), b_held = held(b);
    attend_tile<D, WIDE, KV8>(a, t, p, s_kv, s_ml, &s_others, s_pages, s_masks);
    if (PIECES) return;
    pos = uniform(pos_held), end = uniform(end_held), chunk = uniform(chunk_held), b = uniform(b_held);
  }
}

// More sequences than a cut takes: a tile and KV head per workgroup.
template <int D, bool WIDE, bool KV8>
__global__ __launch_bounds__(WIDE ? 512 : 256, WIDE ? 1 : 2) void tree_attn_many_kernel(const ExtendArgs a) {
  __shared__ __attribute__((aligned(256))) uint16_t s_kv[kTreeLds<D, WIDE, KV8> / 2];
  __shared__ float2 s_ml[(WIDE ? 8 : 4) * 64];
  __shared__ int s_pages[WIDE ? kRingPages : 1];
  __shared__ uint32_t s_masks[kMaskLds<WIDE ? 256 : 32>];
  __shared__ int s_others;
  TileOf t;
  if (!find_tile<WIDE ? 256 : 32>(a, t)) return;
  const TileUnits u = units_of<WIDE, KV8>(min(t.n_rows - t.first, WIDE ? 256 : 32), t.s_b);
  Piece p{(int)blockIdx.x, 0, t.s_b ? u.blocks : 0, true, -1, 0};
  if (threadIdx.x == 0) s_others = 0;
  attend_tile<D, WIDE, KV8>(a, t, p, s_kv, s_ml, &s_others, s_pages, s_masks);
}

// Joins the parts of tiles that several workgroups have taken: D/4 lanes a (row, query head), four outputs each,
// parts in the order of the keys; LANES such take every LANES-th part each and are joined in LDS.
template <int D, int LANES>
__global__ __launch_bounds__(256) void tree_join_kernel(const ExtendArgs a, bool kv8, int tile_rows, int groups) {
  constexpr int L = D / 4, kItems = 256 / (L * LANES), kAhead = 4;
  __shared__ f32x4 s_o[LANES][kItems * L];
  __shared__ float2 s_ml[LANES][kItems * L];
  const int at = threadIdx.x % (kItems * L), lanes = threadIdx.x / (kItems * L);
  const int64_t item = (int64_t)blockIdx.x * kItems + at / L;
  const int e = 4 * (at % L), Hq = a.n_q_heads;
  const int row = (int)(item / Hq), head = (int)(item - (int64_t)row * Hq);
  const bool real = row >= run_offset(a.runs, 0) && row < run_offset(a.runs, a.runs.batch);
  const int note = real ? a.part_n[item] : 0;
  const int g0 = note >> 10 & 1023, n = min(note & 1023, groups - g0);   // (0: written by its only workgroup)
  const int g = head / (Hq / a.n_kv_heads);
  float m = kNegInfF, l = 0.f;
  f32x4 o = {0.f, 0.f, 0.f, 0.f};
  auto fold = [&](const float2& ml, const f32x4& x) {
    const float m_new = fmaxf(m, ml.x), m_use = m_new == kNegInfF ? 0.f : m_new;
    const float f1 = __builtin_amdgcn_exp2f(m - m_use), f2 = __builtin_amdgcn_exp2f(ml.x - m_use);
    m = m_new;
    l = l * f1 + ml.y * f2;
    o = o * f1 + x * f2;
  };
  for (int i0 = lanes; i0 < n; i0 += kAhead * LANES) {
    float2 ml[kAhead];
    f32x4 x[kAhead];
#pragma unroll
    for (int k = 0; k < kAhead; ++k) {   // (past the last part: that one again, not folded)
      const int i = min(i0 + k * LANES, n - 1);
      const size_t part = (2 * ((size_t)(g0 + i) * a.n_kv_heads + g) + (i == 0)) * tile_rows + (note >> 20);
      ml[k] = *reinterpret_cast<const float2*>(a.part_ml + 2 * part);
      x[k] = *reinterpret_cast<const f32x4*>(a.part_o + part * D + e);
    }
#pragma unroll
    for (int k = 0; k < kAhead; ++k)
      if (i0 + k * LANES < n) fold(ml[k], x[k]);
  }
  if constexpr (LANES > 1) {
    s_o[lanes][at] = o;
    s_ml[lanes][at] = make_float2(m, l);
    __syncthreads();
    if (lanes) return;
#pragma unroll
    for (int k = 1; k < LANES; ++k) fold(s_ml[k][at], s_o[k][at]);
  }
  if (n <= 0) return;
  const float v_scale = kv8 && a.v_scale ? a.v_scale[g] : 1.f;
  *reinterpret_cast<u32x2*>(a.out + (size_t)item * D + e) = pack_outputs(o, v_scale, l);
}

template <int D, bool WIDE, bool KV8>
hipError_t launch_d(const TreePlan& p, const ExtendArgs& a, hipStream_t stream) {
  const dim3 block(WIDE ? 512 : 256);
  if (!p.workgroups) {
    hipLaunchKernelGGL((tree_attn_many_kernel<D, WIDE, KV8>), dim3(a.n_kv_heads, p.tiles), block, 0, stream, a);
    return hipGetLastError();
  }
  if (p.pieces) hipLaunchKernelGGL((tree_attn_kernel<D, WIDE, KV8, true>), dim3(p.workgroups), block, 0, stream, a);
  else hipLaunchKernelGGL((tree_attn_kernel<D, WIDE, KV8, false>), dim3(p.workgroups), block, 0, stream, a);
  hipError_t e = hipGetLastError();
  const int groups = p.workgroups / a.n_kv_heads;
  if (e != hipSuccess || groups == 1) return e;
  const int64_t items = (int64_t)a.runs.n_rows * a.n_q_heads;
  auto join = [&](auto kernel, int lanes) {
    const int per = 256 / (D / 4 * lanes);
    hipLaunchKernelGGL(kernel, dim3((unsigned)((items + per - 1) / per)), dim3(256), 0, stream, a, KV8, p.rows, groups);
  };
  // many parts a tile: several times the lanes (a tile has about this many on average)
  if (groups >= 6 * p.tiles) join(tree_join_kernel<D, 8>, 8);
  else join(tree_join_kernel<D, 1>, 1);
  return hipGetLastError();
}

template <int D>
hipError_t launch(const TreePlan& p, bool kv8, const ExtendArgs& a, hipStream_t stream) {
  if (p.rows == 32) return kv8 ? launch_d<D, false, true>(p, a, stream) : launch_d<D, false, false>(p, a, stream);
  return kv8 ? launch_d<D, true, true>(p, a, stream) : launch_d<D, true, false>(p, a, stream);
}

}  // namespace

hipError_t launch_tree_attn(const TreePlan& p, int head_dim, bool kv8, const ExtendArgs& a, hipStream_t stream) {
  return head_dim == 128 ? launch<128>(p, kv8, a, stream) : launch<64>(p, kv8, a, stream);
}

}  // namespace delta
