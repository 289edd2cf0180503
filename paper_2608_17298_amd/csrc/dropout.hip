// Dropout with a mask that is drawn again wherever it is needed, never stored.
//
// Element e (row-major, whatever the strides) is kept iff its 16 random bits
// are >= t; they are half word e % 8 of Philox-4x32-10 (Salmon, Moraes, Dror
// and Shaw, "Parallel random numbers: as easy as 1, 2, 3", 2011) at counter
// (e / 8, offset) under the key seed.  y = residual + (kept ? x s : 0) with
// s = 2^16 / (2^16 - t), so the expectation is exact for the p that is used.
//
// One thread owns one call of the generator, that is 8 consecutive elements:
// 16 bits an element halve the generator's work against a word each (two
// 32x32->64 products and a few adds and xors per round, 10 rounds).  Bound by
// bytes: 1M x 128 bf16 with a residual take 128 us, 6.0 TB/s.
#include "blocks.h"

namespace gart {
namespace {

constexpr int kThreads = 256;
constexpr int kDraw = 8;  // elements per generator call
constexpr int64_t kMaxBlocks = int64_t(1) << 20;

struct Words {
  uint32_t w[4];
};

__device__ __forceinline__ Words philox(uint64_t call, uint64_t offset, uint64_t seed) {
  uint32_t c0 = uint32_t(call), c1 = uint32_t(call >> 32), c2 = uint32_t(offset), c3 = uint32_t(offset >> 32);
  uint32_t k0 = uint32_t(seed), k1 = uint32_t(seed >> 32);
#pragma unroll
  for (int r = 0; r < 10; ++r) {
    const uint64_t p0 = uint64_t(0xD2511F53u) * c0, p1 = uint64_t(0xCD9E8D57u) * c2;
    c0 = uint32_t(p1 >> 32) ^ c1 ^ k0;
    c1 = uint32_t(p1);
    c2 = uint32_t(p0 >> 32) ^ c3 ^ k1;
    c3 = uint32_t(p0);
    k0 += 0x9E3779B9u;
    k1 += 0xBB67AE85u;
  }
  return Words{{c0, c1, c2, c3}};
}

__device__ __forceinline__ bool kept(const Words& w, int j, uint32_t threshold) {
  return ((w.w[j / 2] >> (16 * (j % 2))) & 0xFFFFu) >= threshold;
}

// FLAT: the rows follow one another in x, y and the residual, so the matrix
// is one row (its column count then passes 31 bits).
template <typename T, bool FLAT>
__global__ __launch_bounds__(kThreads) void dropout_kernel(const DropoutArgs a) {
  const T* x = static_cast<const T*>(a.x);  // x, residual and y may be one array: no restrict
  const T* res = static_cast<const T*>(a.residual);
  T* y = static_cast<T*>(a.y);
  constexpr int V = Pack<T>::N;
  const int64_t total = a.rows * a.cols, calls = (total + kDraw - 1) / kDraw;
  for (int64_t b = int64_t(blockIdx.x) * kThreads; b < calls; b += int64_t(gridDim.x) * kThreads) {
    const int64_t call = b + threadIdx.x;
    if (call >= calls) break;
    int64_t row = 0, col = call * kDraw;
    if (!FLAT) {
      const int64_t brow = b * kDraw / a.cols;  // the same for the block
      const uint32_t c = uint32_t(b * kDraw - brow * a.cols) + threadIdx.x * kDraw;
      const uint32_t down = c / uint32_t(a.cols);
      row = brow + down;
      col = c - down * uint32_t(a.cols);
    }
    const Words w = philox(uint64_t(call), a.offset, a.seed);
    if (col + kDraw <= a.cols) {
      const int64_t xo = row * a.x_ld + col, ro = row * a.residual_ld + col, yo = row * a.y_ld + col;
      Pack<T> v[kDraw / V], r[kDraw / V];
#pragma unroll
      for (int q = 0; q < kDraw / V; ++q) {
        v[q] = load_pack(x + xo + q * V);
        if (res) r[q] = load_pack(res + ro + q * V);
      }
#pragma unroll
      for (int q = 0; q < kDraw / V; ++q) {
#pragma unroll
        for (int e = 0; e < V; ++e) {
          float o = kept(w, q * V + e, a.threshold) ? float(v[q].v[e]) * a.scale : 0.0f;
          if (res) o += float(r[q].v[e]);
          v[q].v[e] = T(o);
        }
        store_pack(y + yo + q * V, v[q]);
      }
    } else {  // the draw's elements go on in the next rows, or end with the matrix
      const int count = int(min(int64_t(kDraw), total - call * kDraw));
#pragma unroll
      for (int j = 0; j < kDraw; ++j) {
        if (j < count) {
          float o = kept(w, j, a.threshold) ? float(x[row * a.x_ld + col]) * a.scale : 0.0f;
          if (res) o += float(res[row * a.residual_ld + col]);
          y[row * a.y_ld + col] = T(o);
          if (++col == a.cols) {
            col = 0;
            ++row;
          }
        }
      }
    }
  }
}

// Short strided rows, where few draws stay inside one: a wave draws for 512
// elements, its lanes hand the bits over through LDS and then take every 64th
// element, so that neighbours in memory are neighbours in the wave.
constexpr int kWaveElements = 64 * kDraw;
template <typename T>
__global__ __launch_bounds__(kThreads) void dropout_short_rows_kernel(const DropoutArgs a) {
  __shared__ __attribute__((aligned(16))) uint16_t s_bits[kThreads / 64][kWaveElements];
  const T* x = static_cast<const T*>(a.x);
  const T* res = static_cast<const T*>(a.residual);
  T* y = static_cast<T*>(a.y);
  const int lane = threadIdx.x % 64, wave = threadIdx.x / 64;
  const int64_t total = a.rows * a.cols;
  const uint32_t cols = uint32_t(a.cols), down = 64 / cols, right = 64 % cols;
  uint16_t* bits = s_bits[wave];
  for (int64_t b = int64_t(blockIdx.x) * kThreads * kDraw; b < total; b += int64_t(gridDim.x) * kThreads * kDraw) {
    const int64_t base = b + wave * kWaveElements;
    const Words w = philox(uint64_t(base / kDraw + lane), a.offset, a.seed);
    *reinterpret_cast<uint4*>(bits + lane * kDraw) = make_uint4(w.w[0], w.w[1], w.w[2], w.w[3]);
    __syncthreads();
    const int64_t brow = b / a.cols;  // the same for the block
    const uint32_t c = uint32_t(b - brow * a.cols) + uint32_t(wave * kWaveElements + lane);
    int64_t row = brow + c / cols;
    uint32_t col = c % cols;
#pragma unroll
    for (int q = 0; q < kDraw; ++q) {
      if (base + 64 * q + lane < total) {
        float o = bits[64 * q + lane] >= a.threshold ? float(x[row * a.x_ld + col]) * a.scale : 0.0f;
        if (res) o += float(res[row * a.residual_ld + col]);
        y[row * a.y_ld + col] = T(o);
      }
      row += down;
      col += right;
      if (col >= cols) {
        col -= cols;
        ++row;
      }
    }
    __syncthreads();
  }
}

// Row lengths below which the kernel for short rows is faster (strided rows of 6:
// 11 us against 37, of 33: 18 against 24, of 100: 24.6 against 20.7).
constexpr int64_t kShortRow = 64;

template <typename T>
hipError_t launch(DropoutArgs a, hipStream_t s) {
  if (a.rows <= 0 || a.cols <= 0) return hipSuccess;
  const bool flat = a.rows == 1 || (a.x_ld == a.cols && a.y_ld == a.cols && (!a.residual || a.residual_ld == a.cols));
  if (flat) {
    a.cols *= a.rows;
    a.rows = 1;
  }
  const int64_t blocks = ceil_div64(ceil_div64(a.rows * a.cols, kDraw), kThreads);
  const dim3 grid(uint32_t(blocks < kMaxBlocks ? blocks : kMaxBlocks));
  if (!flat && a.cols % kDraw != 0 && a.cols < kShortRow)
    dropout_short_rows_kernel<T><<<grid, kThreads, 0, s>>>(a);
  else if (flat)
    dropout_kernel<T, true><<<grid, kThreads, 0, s>>>(a);
  else
    dropout_kernel<T, false><<<grid, kThreads, 0, s>>>(a);
  return hipGetLastError();
}

}  // namespace

hipError_t launch_dropout(const DropoutArgs& a, gart_dtype t, hipStream_t s) {
  if (t == GART_DTYPE_F32) return launch<float>(a, s);
  if (t == GART_DTYPE_BF16) return launch<bf16>(a, s);
  return launch<f16>(a, s);
}

}  // namespace gart
