// The linear layer for few rows, a single one above all.  A block takes 16 outputs
// and all rows; its waves share the inputs and read their pieces of 16 weight rows
// straight into fragments, kInFlight at a time, so that a whole block's weights are
// asked for at once.  The waves' sums meet in LDS, in order.  One row of 1024 ->
// 4096 bf16: 4 us, one round trip to memory, launch and joins (8 MB: 2 TB/s).
//
// Every block reads all of x and the whole sum, so it is bound by its own chain of
// inputs, whatever the outputs: few rows with short sums.  Calls against tiles with
// cut sums, us: 16 rows of 1024 -> 1024 f32 7 and 12, of 4096 bf16 10 and 13, but
// of 4096 f32 18 and 16, of 16384 bf16 33 and 19; 64 rows of 1024 -> 1024 bf16 7 and
// 10, but f32 21 and 14, of 4096 -> 256 bf16 21 and 16.
#pragma once

#include <algorithm>

#include "linear.h"

namespace gart {
namespace {

constexpr int kInFlight = 4;
constexpr int kRowsWaves = 16;

// DZ: dz = dl act'(z) in place of y, and g_bias, its sum over the rows.
template <typename T, int MT, bool DZ>
__global__ __launch_bounds__(64 * kRowsWaves) void rows_kernel(const LinearArgs a, T* out, int64_t out_ld,
                                                                 int64_t out_low) {
  constexpr int V = Pack<T>::N, D = kDepth<T>, SIZE = 16 * MT * 16;
  extern __shared__ __attribute__((aligned(16))) float s_acc[];  // [waves][SIZE]
  const int tid = threadIdx.x, lane = tid % 64, wave = tid / 64, waves = blockDim.x / 64;
  const int r = lane % 16, g = lane / 16;
  const int64_t n = int64_t(blockIdx.x) * 16 + r;
  const T* __restrict__ x = static_cast<const T*>(a.x);
  const T* __restrict__ w = static_cast<const T*>(a.w);
  f32x4 acc[MT] = {};
  for (int64_t k0 = int64_t(wave) * D; k0 < a.k; k0 += int64_t(waves) * D * kInFlight) {
    typename Pack<T>::V fw[kInFlight], fx[kInFlight][MT];
#pragma unroll
    for (int u = 0; u < kInFlight; ++u) {
      const int64_t k = k0 + int64_t(u) * waves * D + V * g;
      const int count = int(max(int64_t(0), min(int64_t(V), a.k - k)));
      fw[u] = T(0.0f);
      if (n < a.n && count > 0) fw[u] = load_some(w + n * a.w_ld + k, count).v;
#pragma unroll
      for (int i = 0; i < MT; ++i) {
        fx[u][i] = T(0.0f);
        if (16 * i + r < a.m && count > 0) fx[u][i] = load_some(x + (16 * i + r) * a.x_ld + k, count).v;
      }
    }
#pragma unroll
    for (int u = 0; u < kInFlight; ++u)
#pragma unroll
      for (int i = 0; i < MT; ++i) acc[i] = Mfma<T>::run(fw[u], fx[u][i], acc[i]);
  }
#pragma unroll
  for (int i = 0; i < MT; ++i) *reinterpret_cast<f32x4*>(s_acc + wave * SIZE + (16 * i + r) * 16 + 4 * g) = acc[i];
  __syncthreads();
  const T* bias = static_cast<const T*>(a.bias);
  const T* extra = static_cast<const T*>(DZ ? a.dl : a.residual);
  const int64_t extra_ld = DZ ? a.dl_ld : a.residual_ld;
  for (int o = tid; o < SIZE; o += blockDim.x) {
    const int m = o / 16;
    const int64_t j = int64_t(blockIdx.x) * 16 + o % 16;
    if (m >= a.m || j >= a.n) continue;
    float c = 0.0f;
    for (int v = 0; v < waves; ++v) c += s_acc[v * SIZE + o];
    if (bias) c += float(bias[j]);
    const float e = extra ? float(extra[m * extra_ld + j]) : 0.0f;
    with_activation(a.act, [&](auto act) {
      if constexpr (DZ)
        c = activate_grad<decltype(act)::value>(c, e);
      else
        c = activate<decltype(act)::value>(c) + e;
    });
    T* to = out + m * out_ld + j;
    if (DZ && out_low) {
      if constexpr (sizeof(T) == 2) split_dz<T>(c, *to, to[out_low]);
    } else {
      *to = T(c);
    }
    if (DZ) s_acc[o] = c;  // this thread alone has read it (every wave's share of o)
  }
  if (DZ && a.g_bias) {
    __syncthreads();
    const int64_t j = int64_t(blockIdx.x) * 16 + tid;
    if (tid < 16 && j < a.n) {
      float t = 0.0f;
      for (int m = 0; m < a.m; ++m) t += s_acc[m * 16 + tid];
      static_cast<T*>(a.g_bias)[j] = T(t);
    }
  }
}

template <typename T, bool DZ>
hipError_t rows_launch(const LinearArgs& a, void* out, int64_t out_ld, int64_t out_low, hipStream_t s) {
  if (a.m <= 0 || a.n <= 0) return hipSuccess;
  const int64_t steps = ceil_div64(std::max<int64_t>(a.k, 1), kDepth<T>);
  const int waves = int(std::min<int64_t>(kRowsWaves, ceil_div64(steps, kInFlight)));
  const uint32_t blocks = uint32_t(ceil_div64(a.n, 16));
  const int mt = a.m <= 16 ? 1 : a.m <= 32 ? 2 : 4;
  const size_t bytes = size_t(waves) * mt * 256 * 4;
  T* p = static_cast<T*>(out);
  if (mt == 1)
    rows_kernel<T, 1, DZ><<<blocks, 64 * waves, bytes, s>>>(a, p, out_ld, out_low);
  else if (mt == 2)
    rows_kernel<T, 2, DZ><<<blocks, 64 * waves, bytes, s>>>(a, p, out_ld, out_low);
  else
    rows_kernel<T, 4, DZ><<<blocks, 64 * waves, bytes, s>>>(a, p, out_ld, out_low);
  return hipGetLastError();
}

}  // namespace

template <typename T>
hipError_t rows_forward(const LinearArgs& a, hipStream_t s) {
  return rows_launch<T, false>(a, a.y, a.y_ld, 0, s);
}

template <typename T>
hipError_t rows_dz(const LinearArgs& a, void* dz, int64_t dz_ld, int64_t dz_low, hipStream_t s) {
  return rows_launch<T, true>(a, dz, dz_ld, dz_low, s);
}

}  // namespace gart
