// Sizes and block counts of the streaming forward and backward, shared by
// their launchers and by the scratch they are given.
#pragma once

#include <algorithm>

#include "linear.h"

namespace gart {

// ---- forward ---------------------------------------------------------------------
constexpr int kForwardWaves = 4;
constexpr int kForwardBytes = 64 * 1024;  // of the weight in LDS
constexpr int kForwardBlocks = 2048;

inline int round_inputs(int64_t k) {
  int p = 32;
  while (p < k && p < 512) p *= 2;
  return p;
}

// the weight's rows, 16 bytes longer, and the bias as floats
inline int64_t forward_lds(int kp, int64_t n, size_t es) { return (n + 31) / 32 * 32 * (kp * int64_t(es) + 16 + 4); }

// At most `most` blocks, all with the same number of turns (or one less).
inline int64_t even_blocks(int64_t turns, int64_t most) {
  return turns <= most ? turns : ceil_div64(turns, ceil_div64(turns, most));
}

// ---- backward --------------------------------------------------------------------
// NS: waves side by side over the outputs, 32 each.  With few of them, RG
// groups of NS waves take rows of their own in a tile.  PARTS: dz is in two
// parts (split_dz); what fits LDS with one fits it with two.
template <size_t ES, int KP, int NS, bool PARTS>
struct BackwardSizes {
  static constexpr int RG = NS == 1 ? 4 : NS == 2 ? 2 : 1;
  static constexpr int WAVES = NS * RG, THREADS = 64 * WAVES;
  static constexpr int GROUP_ROWS = NS >= 4 ? 64 : 32, ROWS = GROUP_ROWS * RG;
  static constexpr int NP = 32 * NS;
  static constexpr int PAD = ES == 2 ? 16 : 4;  // spreads rows (and columns' lines) over the banks
  static constexpr int KPITCH = KP + PAD, NPITCH = NP + PAD;
  static constexpr int W = NP * KPITCH, X = ROWS * KPITCH, Z = ROWS * NPITCH;
  static constexpr int Z_LOW = PARTS ? Z : 0;
  static constexpr size_t BYTES = size_t(W + X + Z + Z_LOW) * ES;
  static constexpr bool FITS = BYTES <= 160 * 1024 && KP * int(ES) <= 512;
};

// Blocks: two of four waves for each of the 256 CUs, as many as the registers
// hold where weights are small (100000 x 32 -> 64 f32: three with fewer registers each
// took a tenth longer, four a third).  Of larger weights (64 x 256, 128 x 128 and up
// in 16 bits) a CU holds one, and the n (k + 1) sums that each leaves count: 32000
// rows of 256 -> 128 bf16 write and read 67 MB of them beside 42 MB of rows (63 us,
// in tiles 53; 2000 rows 24 and 30, 100000 rows 98 and 112).
constexpr int64_t kBackwardBlocks = 512;

// All of them, so that CUs get equally many tiles (100000 x 32 -> 64 f32, 1563
// tiles: 27 us; 391 blocks of four turns, on half of the CUs two, 29.5; 36000 x
// 128 -> 100 f32: 72 and 83).
inline int64_t backward_blocks(int64_t tiles) { return std::min(tiles, kBackwardBlocks); }

struct BackwardChoice {
  int kp, ns, rows;  // kp 0: none
};

template <size_t ES, int KP, int NS>
bool offer(int64_t k, int64_t n, BackwardChoice* c) {
  using B = BackwardSizes<ES, KP, NS, false>;
  static_assert(!B::FITS || ES == 4 || BackwardSizes<ES, KP, NS, true>::FITS, "dz in two parts fits");
  if (!B::FITS || k > KP || n > 32 * NS) return false;
  *c = BackwardChoice{KP, NS, B::ROWS};
  return true;
}

template <size_t ES, int KP>
bool offer_inputs(int64_t k, int64_t n, BackwardChoice* c) {
  return offer<ES, KP, 1>(k, n, c) || offer<ES, KP, 2>(k, n, c) || offer<ES, KP, 4>(k, n, c) ||
         offer<ES, KP, 8>(k, n, c);
}

template <size_t ES>
BackwardChoice choose(int64_t k, int64_t n) {
  BackwardChoice c{};
  if (!(offer_inputs<ES, 32>(k, n, &c) || offer_inputs<ES, 64>(k, n, &c) || offer_inputs<ES, 128>(k, n, &c)))
    offer_inputs<ES, 256>(k, n, &c);
  return c;
}

inline BackwardChoice choose_backward(int64_t k, int64_t n, size_t es) {
  return es == 4 ? choose<4>(k, n) : choose<2>(k, n);
}

}  // namespace gart
