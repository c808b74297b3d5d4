// How the tile step of attend_runs.h lays out a workgroup's LDS (no device code: a host test compiles it).
#pragma once

#include <algorithm>

namespace delta {

// Blocks that a ring holds, and the pages that it looks up at a time.
constexpr int kRing = 4, kRingPages = 1024;

// LDS of a body, in bytes: K and V of the blocks, later the outputs of the waves along the keys.
template <int D, int WR, int WK, int KT, bool RING = false, bool KV8 = false>
constexpr int kBodyLds = std::max(RING ? (KV8 ? 2 * 2 * 2 + kRing * 2 : kRing * 2 * 2) * 32 * KT * WK * D
                                       : 2 * (WR == 1 ? 1 : 2) * 32 * KT * WK * D * 2,
                                  WK > 1 ? WR * WK * 64 * D / 2 * 4 : 0);

// A ring of e4m3 blocks of KEYS keys, loaded by NW waves: behind the two buffers of bf16 blocks, the LDS of each
// wave's own loads, 1024 bytes of K and 1024 of V each.  A block of a small head has fewer pieces than the workgroup
// has lanes: then the last waves have no loads and no LDS.
template <int D, int NW, int KEYS>
struct RawRing {
  static constexpr int kPieces = KEYS * D / 16;                    // 16-byte pieces of a block, of K and of V
  static constexpr int kLoads = (kPieces + 64 * NW - 1) / (64 * NW);   // of a wave and block, at most
  static constexpr int kBegin = 2 * 2 * KEYS * D * 2;
  static constexpr bool has(int wave, int load) { return (load * NW + wave) * 64 < kPieces; }
  static constexpr int at(int wave, int stage, int load) {
    return kBegin + ((wave * kRing + stage) * kLoads + load) * 2048;
  }
};

}  // namespace delta
