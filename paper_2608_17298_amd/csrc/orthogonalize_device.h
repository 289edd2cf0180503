// Device code shared by the orthogonalising kernels: what is orthogonalised, numbers
// in two parts, and matrices in the order of the matrix instruction's fragments.
#pragma once

#include "linear.h"
#include "orthogonalize.h"

namespace gart {
namespace {

// ---- the matrix that is orthogonalised ----------------------------------------
// x itself, or of a momentum step u = g + mu m (Nesterov) or m, with m already
// stepped: the same operations wherever it is formed.
template <typename T>
struct Source {
  const T* x;
  int64_t ld;
  const float* m;  // NULL: x itself
  int64_t m_ld;
  float momentum;
  bool nesterov;
};

// A float as high + low.
__device__ __forceinline__ void split(float v, f16& high, f16& low) {
  high = f16(v);
  low = f16(v - float(high));
}

// ---- matrices in the order of fragments ------------------------------------------
// The matrix instruction takes 16 rows by 32 k of an operand, eight consecutive k of
// row r = lane % 16 from k = 8 (lane / 16) in each lane.  X, A and P are stored in
// such blocks, a kilobyte of high parts and one of low parts, side by side along k:
// a wave loads a fragment as it stands, past LDS.  X is stored twice, as itself for
// X X^T and transposed for P X; A and P are symmetric.
struct Blocks {
  f16* data;
  int64_t across;  // blocks along k
  static constexpr int kBlock = 16 * 32, kPair = 2 * kBlock;  // elements
  // the block of rows 16 i and k 32 k
  __device__ __forceinline__ f16* at(int64_t i, int64_t k) const { return data + (i * across + k) * kPair; }
};

// The iteration, with its factors for singular values that start at 1.
struct Iteration {
  float a, b, c, eps;
  int steps;
  Factors of_one;
};

// What `size`, the norm of u, makes of it: the first scale over the norm, and whether
// the steps' factors have to be worked out from where the values start.
__device__ __forceinline__ double first_scale(const Iteration& it, double size, bool& tiny) {
  const double norm = size + double(it.eps);
  tiny = size / norm < kNearOne;  // not if it is a NaN
  return (tiny ? pair_scale(size / norm, kMostX) : double(it.of_one.x)) / norm;
}

}  // namespace
}  // namespace gart
