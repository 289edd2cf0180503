// How the orthogonalising iteration is scaled and laid out.  Plain C++, so that it
// can be asked without a GPU; the scales are also worked out on it.
#pragma once

#include <algorithm>
#include <cmath>
#include <cstdint>

namespace gart {

#ifdef __HIPCC__
#define GART_HOST_DEVICE __host__ __device__
#else
#define GART_HOST_DEVICE
#endif

// X, A = X X^T and P = b A + c A^2 are held as sums of two float16 numbers, high +
// low, both times a power of two that fits the step: off by 2^-22 of an element.
// Singular values of X start at |x| / (|x| + eps) or less, and after each step they
// are values of p(s) = a s + b s^3 + c s^5; so the largest |p| over the interval
// where they lie bounds every element of X, its square those of A, and the largest
// |b t + c t^2| those of P.  With elements times their scale of 2^14 at most, float16
// never overflows (65504), and 2^-24, its smallest number, is 2^-38 of the bound.
//
// |x| is known on the GPU alone.  The bounds are those of a start at 1 unless it is
// below kNearOne, that is unless x is about as small as eps: then the scales are
// worked out there, from where the values start.
constexpr int kMaxSteps = 64;
constexpr double kMaxValue = 0x1p10, kMaxPolynomial = 0x1p60;  // bounds of X and P that steps may reach
constexpr double kNearOne = 0.0625;

struct StepScales {
  double x, a, p;  // powers of two
};

// The power of two by which numbers up to `bound` are multiplied.  Beyond the clamps
// a result of float has nothing left (X; A and P with a small a; 2^-122, where the
// product's last factor ends, counts as nothing), or the matrix adds nothing to a X
// (A and P with |P| below 2^-24 |a|).
GART_HOST_DEVICE inline double pair_scale(double bound, int most) {
  if (!(bound > 0.0)) return 1.0;
  const int e = 13 - ilogb(bound);
  return ldexp(1.0, e > most ? most : e < -60 ? -60 : e);
}
constexpr int kMostX = 120, kMostA = 60, kMostAlone = 120;

GART_HOST_DEVICE inline double larger(double a, double b) { return a > b ? a : b; }

// Scales of the step of values up to bound, and the bound of those after it.
GART_HOST_DEVICE inline double step_scales(double a, double b, double c, double bound, StepScales* out) {
  const double s2 = bound * bound;
  double p = fabs(b * s2 + c * s2 * s2);
  const double top = c != 0.0 ? -b / (2.0 * c) : -1.0;
  if (top > 0.0 && top < s2) p = larger(p, fabs(b * top + c * top * top));
  const int most = fabs(a) < 0x1p24 * p ? kMostAlone : kMostA;
  *out = StepScales{pair_scale(bound, kMostX), pair_scale(s2, most), pair_scale(p, most)};
  if (!(p <= kMaxPolynomial)) return HUGE_VAL;
  // p'(s) = a + 3 b t + 5 c t^2 = 0 with t = s^2
  double next = sqrt(s2) * fabs(a + b * s2 + c * s2 * s2);
  // by the sum that does not cancel, so that a small c (or 0) leaves the root -a / 3b
  double t[2] = {-1.0, -1.0};
  const double disc = 9.0 * b * b - 20.0 * a * c;
  if (disc >= 0.0) {
    const double q = -0.5 * (3.0 * b + copysign(sqrt(disc), b));
    if (c != 0.0) t[0] = q / (5.0 * c);
    if (q != 0.0) t[1] = a / q;
  }
  for (int k = 0; k < 2; ++k)
    if (t[k] > 0.0 && t[k] < s2) next = larger(next, sqrt(t[k]) * fabs(a + b * t[k] + c * t[k] * t[k]));
  return next;
}

// What a step's products are multiplied by, scales included: A = gram (X X^T),
// P = square (A A) + linear A, X = apply (P X) + keep X.
struct StepFactors {
  float gram, none, square, linear, apply, keep;
};

struct Factors {
  float x;  // the first scale of X
  StepFactors step[kMaxSteps];
};

// Of values that start at `bound`; false if they may pass the bounds above.
GART_HOST_DEVICE inline bool step_factors(float a, float b, float c, int steps, double bound, float* x,
                                          StepFactors* out) {
  StepScales s, next;
  bound = step_scales(a, b, c, bound, &s);
  *x = float(s.x);
  for (int k = 0; k < steps; ++k) {
    if (!(bound <= kMaxValue)) return false;
    if (k + 1 < steps)
      bound = step_scales(a, b, c, bound, &next);
    else
      next.x = 1.0;  // the result itself
    out[k] = StepFactors{float(s.a / s.x / s.x), 0.0f, float(c * (s.p / s.a / s.a)), float(b * (s.p / s.a)),
                         float(next.x / s.p / s.x), float(a * (next.x / s.x))};
    s = next;
  }
  return true;
}

// How a product is cut: square tiles of 32, 64 or 128 a block, one block a CU, and
// parts of the sums that a second launch joins.
struct PairCut {
  int side, parts;
  bool symmetric;  // only tiles on and above the diagonal
};
constexpr int64_t kTileSide = 64;
// Launched for them: a triangle with an odd number of rows is folded with one more.
inline int64_t blocks_of(int64_t rows, int64_t cols, int side, bool symmetric) {
  const int64_t i = (rows + side - 1) / side, j = (cols + side - 1) / side, even = i + i % 2;
  return symmetric ? even / 2 * (even + 1) : i * j;
}

// The tiles of a product.  Blocks go to the eight XCDs in turn; each XCD gets a run of
// tiles, of one or two parts of k, that covers a patch of `band` rows, so that its
// cache takes in few rows of both operands.  A triangle of tiles (i <= j) is folded to
// half as many rows: row r, then row n - 1 - r.
struct TileOrder {
  int tiles_i, tiles_j, band;
  bool symmetric;
};
inline TileOrder tile_order(int64_t rows, int64_t cols, int side, bool symmetric) {
  TileOrder o{int((rows + side - 1) / side), int((cols + side - 1) / side), 1, symmetric};
  const int tiles = int(blocks_of(rows, cols, side, symmetric)), most = symmetric ? (o.tiles_i + 1) / 2 : o.tiles_i;
  while (o.band < most && o.band * o.band * 8 < tiles) ++o.band;  // find_tile multiplies it by the columns
  return o;
}
// Tile t of those launched; false where there is none.
GART_HOST_DEVICE inline bool find_tile(const TileOrder& o, int t, int& ti, int& tj) {
  const int n = o.tiles_i, even = n + n % 2;
  const int rows = o.symmetric ? even / 2 : n, cols = o.symmetric ? even + 1 : o.tiles_j;
  const int top = t / (o.band * cols) * o.band, high = o.band < rows - top ? o.band : rows - top;
  const int in = t - top * cols, r = top + in % high, c = in / high;
  ti = r;
  tj = c;
  if (o.symmetric) {
    const bool folded = c >= even - r;
    ti = folded ? even - 1 - r : r;
    tj = folded ? ti + c - (even - r) : r + c;
  }
  return ti < n && tj < o.tiles_j;
}
// Whether the part of a tile from (i0, j0) is a result.  Each wave stores what it has
// formed of a symmetric product on both sides of the diagonal.  A tile on the diagonal
// that several waves share has a part below it: the one above stores that one too, and
// its own sums would not be the same bits, as they add the low parts' products in the
// other order.
GART_HOST_DEVICE inline bool is_result(const TileOrder& o, int64_t rows, int64_t cols, int64_t i0, int64_t j0) {
  return i0 < rows && j0 < cols && !(o.symmetric && i0 > j0);
}

inline PairCut cut_pair(int64_t rows, int64_t cols, int64_t steps, bool symmetric) {
  // measured: us of a block of k for each tile, and of what surrounds the sums
  constexpr int kSides[3] = {32, 64, 128};
  constexpr double kStep[3] = {0.10, 0.20, 0.40}, kAround = 4.0, kJoin = 3.0;
  PairCut best{64, 1, symmetric};
  double least = HUGE_VAL;
  for (int q = 0; q < 3; ++q) {
    const int side = kSides[q];
    const int64_t tiles = blocks_of(rows, cols, side, symmetric);
    const int most = symmetric ? int(std::min<int64_t>(16, std::max<int64_t>(1, steps / 16))) : 1;
    for (int parts = 1; parts <= most; ++parts) {
      const double turns = double((tiles * parts + 255) / 256), length = double((steps + parts - 1) / parts);
      double t = kAround + turns * length * kStep[q];
      if (parts > 1) t += kJoin + double(tiles * parts) * double(side * side) * 2e-6;
      if (t < least) {
        least = t;
        best.side = side;
        best.parts = parts;
      }
    }
  }
  return best;
}
inline size_t partial_floats(int64_t n, int64_t steps) {
  const PairCut c = cut_pair(n, n, steps, true);
  return c.parts == 1 ? 0 : size_t(blocks_of(n, n, c.side, true)) * size_t(c.parts * c.side) * size_t(c.side);
}

// Where things lie in scratch, in bytes; sizes of the padded matrices.
struct MatrixPlan {
  bool tall;            // more rows than columns: X is the transpose
  int64_t n, m;         // the smaller and the larger size
  int64_t n_pad, m_pad;  // multiples of kTileSide
  size_t sums, factors, x[2], xt[2], a, p, total;
};
constexpr int64_t kSumBlocks = 1024;  // partial sums of squares, at most
constexpr int64_t kMostTiles = int64_t(1) << 23;

inline MatrixPlan matrix_plan(int64_t rows, int64_t cols) {
  MatrixPlan p{};
  p.tall = rows > cols;
  p.n = std::min(rows, cols);
  p.m = std::max(rows, cols);
  p.n_pad = (p.n + kTileSide - 1) / kTileSide * kTileSide;
  p.m_pad = (p.m + kTileSide - 1) / kTileSide * kTileSide;
  const size_t x = size_t(p.n_pad) * size_t(p.m_pad) * 4, a = size_t(p.n_pad) * size_t(p.n_pad) * 4;  // two float16
  p.sums = 0;
  p.factors = kSumBlocks * sizeof(double);
  // The X that a step writes is free until then, for the parts of the products before it.
  const size_t partial = 4 * std::max(partial_floats(p.n_pad, p.m_pad / 32), partial_floats(p.n_pad, p.n_pad / 32));
  const size_t both = std::max(2 * x, partial);
  p.x[0] = p.factors + sizeof(StepFactors) * kMaxSteps;
  p.x[1] = p.x[0] + both;
  p.xt[0] = p.x[0] + x;
  p.xt[1] = p.x[1] + x;
  p.a = p.x[1] + both;
  p.p = p.a + a;
  p.total = p.p + a;
  return p;
}

}  // namespace gart
