// Layer norm of a matrix's rows and its gradient.
//
//   d = x - mean(x), rstd = 1 / sqrt(mean(d^2) + eps), h = d rstd, y = h gain + bias
//   w = dl gain:  g_x = rstd (w - mean(w) - h mean(w h));  g_gain = sum of dl h, g_bias = sum of dl over the rows
//
// The variance is formed of the differences from the mean, never as a difference
// of squares.  Nothing of the forward is stored: the gradient reads x anyway and
// forms the statistics again.  Bound by bytes.
#include <algorithm>

#include "blocks.h"

namespace gart {
namespace {

constexpr int kThreads = 256;
constexpr int kWaves = kThreads / 64;
constexpr int64_t kMaxBlocks = int64_t(1) << 20;

// 1 / sqrt(v) by the hardware's instruction, one unit of the last place off, which needs v above the subnormals
__device__ __forceinline__ float rsqrt_of(float v) {
  const bool small = v < 0x1p-100f;
  return __builtin_amdgcn_rsqf(small ? v * 0x1p100f : v) * (small ? 0x1p50f : 1.0f);
}

__device__ __forceinline__ float wave_sum(float v) {
#pragma unroll
  for (int off = 32; off > 0; off >>= 1) v += __shfl_xor(v, off);
  return v;
}

// Sums over the block, the same in every thread; s holds a float per wave and value.
template <int COUNT>
__device__ __forceinline__ void block_sums(float (&v)[COUNT], float (*s)[COUNT]) {
  const int lane = threadIdx.x % 64, wave = threadIdx.x / 64;
#pragma unroll
  for (int q = 0; q < COUNT; ++q) {
    v[q] = wave_sum(v[q]);
    if (lane == 0) s[wave][q] = v[q];
  }
  __syncthreads();
#pragma unroll
  for (int q = 0; q < COUNT; ++q) {
    v[q] = 0.0f;
    for (int w = 0; w < kWaves; ++w) v[q] += s[w][q];
  }
  __syncthreads();
}

// ---- rows of any length: a block a row, read once for each sum -----------------
template <typename T, typename F>
__device__ __forceinline__ void for_packs(int64_t cols, F&& f) {
  for (int64_t c = int64_t(threadIdx.x) * Pack<T>::N; c < cols; c += kThreads * Pack<T>::N)
    f(c, int(min(int64_t(Pack<T>::N), cols - c)));
}

template <typename T>
__device__ __forceinline__ float row_mean(const T* x, int64_t cols, float (*s)[1]) {
  float v[1] = {0.0f};
  for_packs<T>(cols, [&](int64_t c, int count) {
    const Pack<T> p = load_some(x + c, count);
#pragma unroll
    for (int e = 0; e < Pack<T>::N; ++e) v[0] += float(p.v[e]);
  });
  block_sums(v, s);
  return v[0] / float(cols);
}

template <typename T>
__global__ __launch_bounds__(kThreads) void long_rows_kernel(const LayerNormArgs a) {
  __shared__ float s[kWaves][1];
  const T* gain = static_cast<const T*>(a.gain);
  const T* bias = static_cast<const T*>(a.bias);
  for (int64_t row = blockIdx.x; row < a.rows; row += gridDim.x) {
    const T* x = static_cast<const T*>(a.x) + row * a.x_ld;
    T* y = static_cast<T*>(a.y) + row * a.y_ld;
    const float mean = row_mean(x, a.cols, s);
    float v[1] = {0.0f};
    for_packs<T>(a.cols, [&](int64_t c, int count) {
      const Pack<T> p = load_some(x + c, count);
#pragma unroll
      for (int e = 0; e < Pack<T>::N; ++e) {
        const float d = float(p.v[e]) - mean;
        if (e < count) v[0] = fmaf(d, d, v[0]);
      }
    });
    block_sums(v, s);
    const float rstd = rsqrt_of(v[0] / float(a.cols) + a.eps);
    for_packs<T>(a.cols, [&](int64_t c, int count) {  // y may be x: every element is its own thread's
      Pack<T> p = load_some(x + c, count), g, b;
      if (gain) g = load_some(gain + c, count);
      if (bias) b = load_some(bias + c, count);
#pragma unroll
      for (int e = 0; e < Pack<T>::N; ++e) {
        float h = (float(p.v[e]) - mean) * rstd;
        if (gain) h *= float(g.v[e]);
        if (bias) h += float(b.v[e]);
        p.v[e] = T(h);
      }
      store_some(y + c, p, count);
    });
  }
}

// g_x, and the rows' mean and rstd for the column sums
template <typename T>
__global__ __launch_bounds__(kThreads) void long_rows_grad_kernel(const LayerNormArgs a, float2* __restrict__ stats) {
  __shared__ float s1[kWaves][1], s3[kWaves][3];
  const T* gain = static_cast<const T*>(a.gain);
  for (int64_t row = blockIdx.x; row < a.rows; row += gridDim.x) {
    const T* x = static_cast<const T*>(a.x) + row * a.x_ld;
    const T* dl = static_cast<const T*>(a.dl) + row * a.dl_ld;
    const float mean = row_mean(x, a.cols, s1), n = float(a.cols);
    float v[3] = {0.0f, 0.0f, 0.0f};  // d^2, w, w d
    for_packs<T>(a.cols, [&](int64_t c, int count) {
      const Pack<T> p = load_some(x + c, count), q = load_some(dl + c, count);
      Pack<T> g;
      if (gain) g = load_some(gain + c, count);
#pragma unroll
      for (int e = 0; e < Pack<T>::N; ++e) {
        if (e >= count) continue;
        const float d = float(p.v[e]) - mean, w = gain ? float(q.v[e]) * float(g.v[e]) : float(q.v[e]);
        v[0] = fmaf(d, d, v[0]);
        v[1] += w;
        v[2] = fmaf(w, d, v[2]);
      }
    });
    block_sums(v, s3);
    const float rstd = rsqrt_of(v[0] / n + a.eps), mw = v[1] / n, along = v[2] / n * rstd;
    if (stats && threadIdx.x == 0) stats[row] = make_float2(mean, rstd);
    if (!a.g_x) continue;
    T* g_x = static_cast<T*>(a.g_x) + row * a.g_x_ld;
    for_packs<T>(a.cols, [&](int64_t c, int count) {
      Pack<T> p = load_some(x + c, count), q = load_some(dl + c, count), g;
      if (gain) g = load_some(gain + c, count);
#pragma unroll
      for (int e = 0; e < Pack<T>::N; ++e) {
        const float h = (float(p.v[e]) - mean) * rstd, w = gain ? float(q.v[e]) * float(g.v[e]) : float(q.v[e]);
        p.v[e] = T(rstd * (w - mw - h * along));
      }
      store_some(g_x + c, p, count);
    });
  }
}

// Sums over one part of the rows, for 64 columns a block: sums[part] = [g_gain, g_bias]
template <typename T>
__global__ __launch_bounds__(kThreads) void column_grads_kernel(const LayerNormArgs a, const float2* __restrict__ stats,
                                                                int64_t part, float* __restrict__ sums) {
  __shared__ float s[kWaves][2][64];
  const int lane = threadIdx.x % 64, wave = threadIdx.x / 64;
  const int64_t r0 = int64_t(blockIdx.x) * part, r1 = min(a.rows, r0 + part);
  for (int64_t j0 = int64_t(blockIdx.y) * 64; j0 < a.cols; j0 += int64_t(gridDim.y) * 64) {
    const int64_t j = j0 + lane;
    float gain = 0.0f, bias = 0.0f;
    if (j < a.cols)
      for (int64_t r = r0 + wave; r < r1; r += kWaves) {
        const float dl = float(static_cast<const T*>(a.dl)[r * a.dl_ld + j]);
        const float2 st = stats[r];
        gain = fmaf(dl, (float(static_cast<const T*>(a.x)[r * a.x_ld + j]) - st.x) * st.y, gain);
        bias += dl;
      }
    s[wave][0][lane] = gain;
    s[wave][1][lane] = bias;
    __syncthreads();
    if (wave < 2 && j < a.cols)
      sums[(int64_t(blockIdx.x) * 2 + wave) * a.cols + j] =
          (s[0][wave][lane] + s[1][wave][lane]) + (s[2][wave][lane] + s[3][wave][lane]);
    __syncthreads();
  }
}

// g_gain and g_bias (either may be NULL) from the parts' sums
constexpr int kJoinWaves = 16;
template <typename T>
__global__ __launch_bounds__(64 * kJoinWaves) void join_column_grads_kernel(const float* __restrict__ sums,
                                                                            int64_t parts, int64_t cols,
                                                                            T* __restrict__ g_gain,
                                                                            T* __restrict__ g_bias) {
  __shared__ float s[kJoinWaves][64];
  const int lane = threadIdx.x % 64, wave = threadIdx.x / 64;
  for (int64_t b = int64_t(blockIdx.x) * 64; b < 2 * cols; b += int64_t(gridDim.x) * 64) {
    const int64_t e = b + lane;
    T* to = e < cols ? g_gain : g_bias;
    float t = 0.0f;
    if (e < 2 * cols && to)
      for (int64_t p = wave; p < parts; p += kJoinWaves) t += sums[p * 2 * cols + e];
    s[wave][lane] = t;
    __syncthreads();
    if (wave == 0 && e < 2 * cols && to) {
#pragma unroll
      for (int w = 1; w < kJoinWaves; ++w) t += s[w][lane];
      to[e < cols ? e : e - cols] = T(t);
    }
    __syncthreads();
  }
}

constexpr int64_t kPartRows = 256, kMaxParts = 512;
struct Plan {
  int64_t part, parts;
  size_t stats, total;
};
Plan plan_of(int64_t rows, int64_t cols) {
  Plan p{};
  p.part = std::max(kPartRows, ceil_div64(rows, kMaxParts));
  p.parts = ceil_div64(rows, p.part);
  p.stats = size_t(ceil_div64(p.parts * 2 * cols * 4, 16)) * 16;
  p.total = p.stats + size_t(rows) * sizeof(float2);
  return p;
}

template <typename T>
hipError_t forward(const LayerNormArgs& a, hipStream_t s) {
  if (a.rows <= 0 || a.cols <= 0) return hipSuccess;
  long_rows_kernel<T><<<uint32_t(std::min(a.rows, kMaxBlocks)), kThreads, 0, s>>>(a);
  return hipGetLastError();
}

template <typename T>
hipError_t backward(const LayerNormArgs& a, hipStream_t s) {
  if (a.cols <= 0) return hipSuccess;
  const Plan p = plan_of(a.rows, a.cols);
  const bool columns = a.g_gain || a.g_bias;
  float* sums = static_cast<float*>(a.scratch);
  float2* stats = reinterpret_cast<float2*>(static_cast<char*>(a.scratch) + p.stats);
  hipError_t e = hipSuccess;
  if (a.rows > 0 && (a.g_x || columns)) {
    long_rows_grad_kernel<T><<<uint32_t(std::min(a.rows, kMaxBlocks)), kThreads, 0, s>>>(a, columns ? stats : nullptr);
    if ((e = hipGetLastError()) != hipSuccess) return e;
  }
  if (!columns) return e;
  const int64_t groups = ceil_div64(a.cols, 64);
  if (p.parts > 0) {
    const dim3 grid(uint32_t(p.parts), uint32_t(std::min<int64_t>(groups, 65535)));
    column_grads_kernel<T><<<grid, kThreads, 0, s>>>(a, stats, p.part, sums);
    if ((e = hipGetLastError()) != hipSuccess) return e;
  }
  const int64_t blocks = std::min<int64_t>(ceil_div64(2 * a.cols, 64), 1 << 16);
  join_column_grads_kernel<T><<<uint32_t(blocks), 64 * kJoinWaves, 0, s>>>(
      sums, p.parts, a.cols, static_cast<T*>(a.g_gain), static_cast<T*>(a.g_bias));
  return hipGetLastError();
}

}  // namespace

size_t layer_norm_backward_scratch_bytes(int64_t rows, int64_t cols, gart_dtype) {
  if (rows <= 0 || cols <= 0) return 0;
  return plan_of(rows, cols).total;
}

hipError_t launch_layer_norm(const LayerNormArgs& a, gart_dtype t, hipStream_t s) {
  if (t == GART_DTYPE_F32) return forward<float>(a, s);
  if (t == GART_DTYPE_BF16) return forward<bf16>(a, s);
  return forward<f16>(a, s);
}

hipError_t launch_layer_norm_backward(const LayerNormArgs& a, gart_dtype t, hipStream_t s) {
  if (t == GART_DTYPE_F32) return backward<float>(a, s);
  if (t == GART_DTYPE_BF16) return backward<bf16>(a, s);
  return backward<f16>(a, s);
}

}  // namespace gart
