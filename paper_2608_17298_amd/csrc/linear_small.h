// The linear layer's gradient where rows times outputs are few, in 16 bits.
//
// Two launches, bound by their latency: a wave per element of dz, which stays
// float, then both products.  Short sums take 512 columns of four rows a wave; long
// ones a block per 64 columns of a row, whose waves share the sum and join in LDS,
// in order.
//
// A call from Python, silu in bf16, against the kernels for larger sizes: 1000 rows
// of 1000 -> 1 15 us and 34, 300 x 2000 -> 3 12 and 30, one row of 1024 -> 1000 13
// and 17, 8 x 200 -> 100 12 and 21, 64 x 1000 -> 16 12 and 14; above 1024 elements
// of dz 500 x 300 -> 4 12 and 33, but 64 x 1000 -> 32 18 and 14.  One streaming block
// is faster while the weight it reads and writes alone is small: 1 x 32 -> 64 12 and
// 10, 16 x 64 -> 48 14 and 10, 32 x 128 -> 32 24 and 12, 8 x 128 -> 64 12 and 11; with
// 128 x 128 weights 12 and 16, with 256 inputs (1 -> 32) 12 and 20.
#pragma once

#include <algorithm>

#include "linear.h"

namespace gart {
namespace {

constexpr int kSmallDzWaves = 4;

// dz [m, n], without gaps
template <typename T>
__global__ __launch_bounds__(64 * kSmallDzWaves) void small_dz_kernel(const LinearArgs a, float* __restrict__ dz) {
  constexpr int V = Pack<T>::N;
  const int lane = threadIdx.x % 64;
  const int64_t e = int64_t(blockIdx.x) * kSmallDzWaves + threadIdx.x / 64;
  if (e >= a.m * a.n) return;
  const int64_t r = e / a.n, j = e - r * a.n;
  const T* x = static_cast<const T*>(a.x) + r * a.x_ld;
  const T* w = static_cast<const T*>(a.w) + j * a.w_ld;
  float z = 0.0f;
  for (int64_t c = lane * V; c < a.k; c += 64 * V) {
    const int count = int(min(int64_t(V), a.k - c));
    const Pack<T> px = load_some(x + c, count), pw = load_some(w + c, count);
#pragma unroll
    for (int i = 0; i < V; ++i) z = fmaf(float(px.v[i]), float(pw.v[i]), z);
  }
#pragma unroll
  for (int off = 1; off < 64; off <<= 1) z += __shfl_xor(z, off);
  if (lane > 0) return;
  if (a.bias) z += float(static_cast<const T*>(a.bias)[j]);
  const float dl = float(static_cast<const T*>(a.dl)[r * a.dl_ld + j]);
  with_activation(a.act, [&](auto act) { dz[e] = activate_grad<decltype(act)::value>(z, dl); });
}

// One of the products dz W (g_x) and dz^T x (g_weight): rows x k outputs, sums of
// `terms` rows of p times dz[row * dz_row + i * dz_step].
struct SmallSide {
  const void* p;
  void* out;  // may be NULL
  int64_t ld, out_ld, rows, terms, dz_row, dz_step, blocks;
};
constexpr int kFewTerms = 32;  // more are shared by a block's waves; rows are then fewer
constexpr int kSmallRows = 4;  // a wave's, where terms are few

// g_bias (may be NULL): a sum over the terms of each row of the second side.
template <typename T>
__global__ __launch_bounds__(1024) void small_grad_kernel(const SmallSide sx, const SmallSide sw, int64_t k,
                                                          const float* __restrict__ dz, T* __restrict__ g_bias) {
  constexpr int V = Pack<T>::N;
  __shared__ float s[16][64];
  const int lane = threadIdx.x % 64, wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64), waves = blockDim.x / 64;
  const bool second = blockIdx.x >= sx.blocks;
  const SmallSide& g = second ? sw : sx;
  const int64_t b = second ? blockIdx.x - sx.blocks : blockIdx.x;
  const T* p = static_cast<const T*>(g.p);
  T* out = static_cast<T*>(g.out);
  if (g.terms <= kFewTerms) {  // a pack of columns a lane, kSmallRows rows a wave
    const int64_t across = (k + 64 * V - 1) / (64 * V), c = (b % across * 64 + lane) * V;
    const int64_t row0 = (b / across * waves + wave) * kSmallRows;
    const int count = int(max(int64_t(0), min(int64_t(V), k - c)));
    if (out && count > 0) {
      float t[kSmallRows][V] = {};
#pragma unroll 4
      for (int64_t i = 0; i < g.terms; ++i) {
        const Pack<T> v = load_some(p + i * g.ld + c, count);
#pragma unroll
        for (int q = 0; q < kSmallRows; ++q) {
          const float d = dz[min(row0 + q, g.rows - 1) * g.dz_row + i * g.dz_step];
#pragma unroll
          for (int e = 0; e < V; ++e) t[q][e] = fmaf(d, float(v.v[e]), t[q][e]);
        }
      }
#pragma unroll
      for (int q = 0; q < kSmallRows; ++q) {
        if (row0 + q >= g.rows) continue;
        Pack<T> o;
#pragma unroll
        for (int e = 0; e < V; ++e) o.v[e] = T(t[q][e]);
        store_some(out + (row0 + q) * g.out_ld + c, o, count);
      }
    }
    if (second && g_bias && b % across == 0 && lane < kSmallRows && row0 + lane < g.rows) {
      float t = 0.0f;
      for (int64_t i = 0; i < g.terms; ++i) t += dz[(row0 + lane) * g.dz_row + i * g.dz_step];
      g_bias[row0 + lane] = T(t);
    }
    return;
  }
  // a row and 64 columns a block
  const int64_t across = (k + 63) / 64, c = b % across * 64 + lane, row = b / across;
  const float* d = dz + row * g.dz_row;
  if (out) {
    float t = 0.0f;
    if (c < k) {
#pragma unroll 8
      for (int64_t i = wave; i < g.terms; i += waves) t = fmaf(d[i * g.dz_step], float(p[i * g.ld + c]), t);
    }
    s[wave][lane] = t;
    __syncthreads();
    if (wave == 0 && c < k) {
      for (int v = 1; v < waves; ++v) t += s[v][lane];
      out[row * g.out_ld + c] = T(t);
    }
  }
  if (second && g_bias && b % across == 0 && wave == waves - 1) {
    float t = 0.0f;
    for (int64_t i = lane; i < g.terms; i += 64) t += d[i * g.dz_step];
#pragma unroll
    for (int off = 1; off < 64; off <<= 1) t += __shfl_xor(t, off);
    if (lane == 0) g_bias[row] = T(t);
  }
}

template <typename T>
hipError_t small_backward(const LinearArgs& a, float* dz, hipStream_t s) {
  small_dz_kernel<T><<<uint32_t(ceil_div64(a.m * a.n, kSmallDzWaves)), 64 * kSmallDzWaves, 0, s>>>(a, dz);
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;
  const int waves = std::max(a.m, a.n) > kFewTerms ? 16 : 4;
  auto blocks = [&](int64_t rows, int64_t terms) {
    return terms <= kFewTerms ? ceil_div64(rows, kSmallRows * waves) * ceil_div64(a.k, 64 * Pack<T>::N)
                              : rows * ceil_div64(a.k, 64);
  };
  const SmallSide sx{a.w, a.g_x, a.w_ld, a.g_x_ld, a.m, a.n, a.n, 1, a.g_x ? blocks(a.m, a.n) : 0};
  const SmallSide sw{a.x, a.g_w, a.x_ld, a.g_w_ld, a.n, a.m, 1, a.n, a.g_w || a.g_bias ? blocks(a.n, a.m) : 0};
  if (sx.blocks + sw.blocks == 0) return hipSuccess;
  small_grad_kernel<T><<<uint32_t(sx.blocks + sw.blocks), 64 * waves, 0, s>>>(sx, sw, a.k, dz,
                                                                            static_cast<T*>(a.g_bias));
  return hipGetLastError();
}

}  // namespace
}  // namespace gart
