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
#include "linear.h"

namespace gart {
namespace {

constexpr int kThreads = 256;
constexpr int kWaves = kThreads / 64;
constexpr int64_t kMaxBlocks = int64_t(1) << 20;

// 1 / sqrt(v) by the hardware's instruction, which needs v above the subnormals and is
// a unit of the last place off, the same for a whole row, and a step of Newton's.
__device__ __forceinline__ float rsqrt_of(float v) {
  const bool small = v < 0x1p-100f;
  if (small) v *= 0x1p100f;
  const float r = __builtin_amdgcn_rsqf(v), e = fmaf(-(v * r), r, 1.0f);
  const float q = e == e ? fmaf(0.5f * r, e, r) : r;  // of 0 and infinity as it is
  return small ? q * 0x1p50f : q;
}

// s / n by n's reciprocal, the quotient set right by its own remainder: exact where
// it is a float, as the mean of a row of one value has to be, in a fourth of the
// division's instructions.  An infinite s stays.
struct Count {
  float n, inv;
  __device__ __forceinline__ explicit Count(int64_t c) : n(float(c)), inv(1.0f / float(c)) {}
  __device__ __forceinline__ float mean(float s) const {
    const float q = s * inv, r = fmaf(-q, n, s);
    return r == r ? fmaf(r, inv, q) : q;
  }
};

// Sums over groups of G neighbouring lanes, the same bits in all of them: each
// step adds what a lane's partner holds.  Up to 16 lanes the partner's value comes
// with the addition (DPP: quads, half rows and rows mirrored); halves of 32 and of
// 64 trade places by the swapping moves.
template <int CTRL>
__device__ __forceinline__ float add_dpp(float v) {
  const int o = __builtin_amdgcn_update_dpp(0, __builtin_bit_cast(int, v), CTRL, 0xF, 0xF, true);
  return v + __builtin_bit_cast(float, o);
}
template <int G>
__device__ __forceinline__ float group_sum(float v) {
  if constexpr (G >= 2) v = add_dpp<0xB1>(v);    // lanes 1 0 3 2 of each quad
  if constexpr (G >= 4) v = add_dpp<0x4E>(v);    // lanes 2 3 0 1
  if constexpr (G >= 8) v = add_dpp<0x141>(v);   // half row mirrored
  if constexpr (G >= 16) v = add_dpp<0x140>(v);  // row mirrored
  if constexpr (G >= 32) {
    const uint32_t w = __builtin_bit_cast(uint32_t, v);
    const auto p = __builtin_amdgcn_permlane16_swap(w, w, false, false);
    const uint32_t x = p[0], y = p[1];
    v = __builtin_bit_cast(float, x) + __builtin_bit_cast(float, y);
  }
  if constexpr (G >= 64) {
    const uint32_t w = __builtin_bit_cast(uint32_t, v);
    const auto p = __builtin_amdgcn_permlane32_swap(w, w, false, false);
    const uint32_t x = p[0], y = p[1];
    v = __builtin_bit_cast(float, x) + __builtin_bit_cast(float, y);
  }
  return v;
}

// Sums over the block, the same in every thread; s holds a float per wave and value.
template <int COUNT, int WAVES>
__device__ __forceinline__ void block_sums(float (&v)[COUNT], float (&s)[WAVES][COUNT]) {
  const int lane = threadIdx.x % 64, wave = threadIdx.x / 64;
#pragma unroll
  for (int q = 0; q < COUNT; ++q) {
    v[q] = group_sum<64>(v[q]);
    if (lane == 0) s[wave][q] = v[q];
  }
  lds_barrier();
#pragma unroll
  for (int q = 0; q < COUNT; ++q) {
    v[q] = s[0][q];
#pragma unroll
    for (int w = 1; w < WAVES; ++w) v[q] += s[w][q];
    asm volatile("" : "+v"(v[q]));  // read before the barrier, also where the sum is used in a branch alone
  }
  lds_barrier();
}

// ---- rows that registers hold ---------------------------------------------------
// A row belongs to a group of lanes that hold U packs each, the group's first packs
// side by side.  The last pack of a row ends with the row and overlaps the one
// before; what it holds of that counts once (`skip` leading elements do not, by a
// weight of 0: they are the row's, so a NaN among them is the row's as well) and is
// stored twice with the same value.  Rows shorter than a pack are a lane's.
enum RowEnd {
  END_EXACT,  // whole packs, one for each lane
  END_SHARED,
  END_TINY
};

template <typename T, int U, RowEnd END>
struct RowPacks {
  static constexpr int V = Pack<T>::N;
  int at[U], skip[U];
  int cols;
  float weight[U][V];  // of the packs that may not be full
  // lanes of the group, and this one's place in it
  __device__ __forceinline__ RowPacks(int cols, int lanes, int lane) : cols(cols) {
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int c = (u * lanes + lane) * V;
      at[u] = END == END_SHARED ? min(c, cols - V) : c;
      skip[u] = END == END_SHARED ? c - at[u] : 0;
#pragma unroll
      for (int e = 0; e < V; ++e) weight[u][e] = (END == END_TINY ? e < cols : e >= skip[u]) ? 1.0f : 0.0f;
    }
  }
  // Groups with two or three packs a lane are chosen for rows that reach the lanes'
  // last ones (with_lanes, with_block).
  static __device__ __forceinline__ constexpr bool full(int u) {
    return END == END_EXACT || (END == END_SHARED && U <= 3 && u < U - 1);
  }
  __device__ __forceinline__ bool on(int u) const { return END != END_SHARED || full(u) || skip[u] < V; }
  __device__ __forceinline__ bool counts(int u, int e) const {
    return full(u) || (END == END_SHARED ? e >= skip[u] : e < cols);
  }
  __device__ __forceinline__ float weighed(int u, int e, float v) const { return full(u) ? v : v * weight[u][e]; }
  __device__ __forceinline__ float add(int u, int e, float v, float t) const {
    return full(u) ? t + v : fmaf(v, weight[u][e], t);
  }
  __device__ __forceinline__ Pack<T> load(const T* row, int u) const {
    return END == END_TINY ? load_some(row, cols) : load_pack(row + at[u]);
  }
  __device__ __forceinline__ void store(T* row, int u, const Pack<T>& p) const {
    if (END == END_TINY)
      store_some(row, p, cols);
    else if (on(u))
      store_pack(row + at[u], p);
  }
  // gain or bias, or `none` in its place: a choice for each element would cost more than its product
  __device__ __forceinline__ void load_or(Pack<T> (&p)[U], const T* from, float none) const {
#pragma unroll
    for (int u = 0; u < U; ++u) {
      if (from)
        p[u] = load(from, u);
      else
        p[u].v = T(none);
    }
  }
  // this lane's sums of the elements, and of their squared distances from the mean
  __device__ __forceinline__ float sum(const Pack<T> (&x)[U]) const {
    float t = 0.0f;
#pragma unroll
    for (int u = 0; u < U; ++u)
#pragma unroll
      for (int e = 0; e < V; ++e) t = add(u, e, float(x[u].v[e]), t);
    return t;
  }
  __device__ __forceinline__ float squares(const Pack<T> (&x)[U], float mean) const {
    float t = 0.0f;
#pragma unroll
    for (int u = 0; u < U; ++u)
#pragma unroll
      for (int e = 0; e < V; ++e) {
        const float d = float(x[u].v[e]) - mean;
        t = fmaf(weighed(u, e, d), d, t);
      }
    return t;
  }
};

// G lanes a row, U packs each, so that a row is read once and no wave waits for another.
// The next row is on its way while one is worked on.  Bound by bytes: 1M x 32 f32 in
// 47 us, 5.4 TB/s (a large copy reaches 5.0).
template <typename T, int G, int U, RowEnd END>
__global__ __launch_bounds__(kThreads, U == 1 ? 8 : 3) void rows_kernel(const LayerNormArgs a) {
  constexpr int V = Pack<T>::N, ROWS = kThreads / G;
  const RowPacks<T, U, END> at(int(a.cols), G, threadIdx.x % G);
  const T* gain = static_cast<const T*>(a.gain);
  const T* bias = static_cast<const T*>(a.bias);
  Pack<T> g[U], b[U], x[U];
  at.load_or(g, gain, 1.0f);
  at.load_or(b, bias, 0.0f);
  const Count n(a.cols);
  const int64_t step = int64_t(gridDim.x) * ROWS;
  int64_t row = int64_t(blockIdx.x) * ROWS + threadIdx.x / G;
  auto load = [&](int64_t r) {
    const T* p = static_cast<const T*>(a.x) + min(r, a.rows - 1) * a.x_ld;
#pragma unroll
    for (int u = 0; u < U; ++u) x[u] = at.load(p, u);
  };
  load(row);
  for (int64_t first = int64_t(blockIdx.x) * ROWS; first < a.rows; first += step, row += step) {
    const float mean = n.mean(group_sum<G>(at.sum(x)));
    const float rstd = rsqrt_of(n.mean(group_sum<G>(at.squares(x, mean))) + a.eps);
    Pack<T> y[U];
#pragma unroll
    for (int u = 0; u < U; ++u)
#pragma unroll
      for (int e = 0; e < V; ++e) {
        const float h = (float(x[u].v[e]) - mean) * rstd;
        y[u].v[e] = T(fmaf(h, float(g[u].v[e]), float(b[u].v[e])));
      }
    if (first + step < a.rows) load(row + step);  // before the stores, which it would wait for
    if (row < a.rows) {
      T* p = static_cast<T*>(a.y) + row * a.y_ld;
#pragma unroll
      for (int u = 0; u < U; ++u) at.store(p, u, y[u]);
    }
  }
}

// A block a row, for rows past what a wave holds; the other blocks of a CU read while
// one waits for its sums.  Bound by bytes: 8191 x 4096 f16 in 28 us, 4.8 TB/s.  Eight
// f16 packs a thread of 512 spill 24 registers (4000 x 32768 f16 185 us, bf16 124).
template <typename T, int THREADS, int U>
__global__ __launch_bounds__(THREADS) void block_rows_kernel(const LayerNormArgs a) {
  constexpr int V = Pack<T>::N;
  __shared__ float s[2][THREADS / 64][1];
  const RowPacks<T, U, END_SHARED> at(int(a.cols), THREADS, threadIdx.x);
  const T* gain = static_cast<const T*>(a.gain);
  const T* bias = static_cast<const T*>(a.bias);
  const Count n(a.cols);
  for (int64_t row = blockIdx.x; row < a.rows; row += gridDim.x) {
    const T* p = static_cast<const T*>(a.x) + row * a.x_ld;
    Pack<T> x[U], g[U], b[U];
#pragma unroll
    for (int u = 0; u < U; ++u) x[u] = at.load(p, u);
    at.load_or(g, gain, 1.0f);
    at.load_or(b, bias, 0.0f);
    auto sum = [&](float v, int h) {
      float w[1] = {v};
      block_sums(w, s[h]);
      return w[0];
    };
    const float mean = n.mean(sum(at.sum(x), 0));
    const float rstd = rsqrt_of(n.mean(sum(at.squares(x, mean), 1)) + a.eps);
    T* q = static_cast<T*>(a.y) + row * a.y_ld;
#pragma unroll
    for (int u = 0; u < U; ++u) {
#pragma unroll
      for (int e = 0; e < V; ++e) {
        const float h = (float(x[u].v[e]) - mean) * rstd;
        x[u].v[e] = T(fmaf(h, float(g[u].v[e]), float(b[u].v[e])));
      }
      at.store(q, u, x[u]);
    }
  }
}

// The gradient: THREADS / G rows at a time, or one of a whole block (G = THREADS).
// COLUMNS: lanes add dl h and dl of their columns up over the rows that the block takes,
// and the block leaves its sums in sums[block] = [g_gain, g_bias], or, alone, the
// result.  Else sums, if it is not NULL, takes the rows' mean and rstd.
// Bound by bytes in large calls, 1M x 64 f32 in 146 us with the join, 5.3 TB/s; where a
// block has a few turns, by them and the join in LDS: 8191 x 1023 bf16 in 14 us.
template <typename T, int G, int U, RowEnd END, int THREADS, bool COLUMNS>
__global__ __launch_bounds__(THREADS) void rows_grad_kernel(const LayerNormArgs a, float* __restrict__ sums) {
  constexpr int V = Pack<T>::N, ROWS = THREADS / G, WAVES = THREADS / 64;
  constexpr bool BLOCK = G > 64;
  __shared__ float s1[BLOCK ? WAVES : 1][1], s3[BLOCK ? WAVES : 1][3];
  __shared__ float s_join[BLOCK ? 1 : WAVES][BLOCK ? 1 : G * V];
  const int lane = threadIdx.x % G;
  const RowPacks<T, U, END> at(int(a.cols), G, lane);
  const T* gain = static_cast<const T*>(a.gain);
  Pack<T> g[U], x[U], dl[U];
  at.load_or(g, gain, 1.0f);
  float g_gain[COLUMNS ? U : 1][V] = {}, g_bias[COLUMNS ? U : 1][V] = {};
  const Count n(a.cols);
  const int64_t step = int64_t(gridDim.x) * ROWS;
  int64_t row = int64_t(blockIdx.x) * ROWS + threadIdx.x / G;
  auto load = [&](int64_t r) {
    r = min(r, a.rows - 1);
    const T* p = static_cast<const T*>(a.x) + r * a.x_ld;
    const T* q = static_cast<const T*>(a.dl) + r * a.dl_ld;
#pragma unroll
    for (int u = 0; u < U; ++u) {
      x[u] = at.load(p, u);
      dl[u] = at.load(q, u);
    }
  };
  load(row);
  for (int64_t first = int64_t(blockIdx.x) * ROWS; first < a.rows; first += step, row += step) {
    float m[1] = {at.sum(x)};
    if constexpr (BLOCK)
      block_sums(m, s1);
    else
      m[0] = group_sum<G>(m[0]);
    const float mean = n.mean(m[0]);
    // With more than eight elements a lane, packs are converted again where they are
    // used: kept as floats through the sums they would take too many registers.
    auto renew = [&]() {
      if constexpr (sizeof(T) == 2 && U > 1) {
#pragma unroll
        for (int u = 0; u < U; ++u) {
          arrive(x[u].v);
          arrive(dl[u].v);
          arrive(g[u].v);
        }
      }
    };
    renew();
    auto weighted = [&](int u, int e) { return float(dl[u].v[e]) * float(g[u].v[e]); };
    float v[3] = {0.0f, 0.0f, 0.0f};  // d^2, w, w d
#pragma unroll
    for (int u = 0; u < U; ++u)
#pragma unroll
      for (int e = 0; e < V; ++e) {
        // a choice, no weight: an infinite dl makes no NaN of its row
        const float d = float(x[u].v[e]) - mean, w = at.counts(u, e) ? weighted(u, e) : 0.0f;
        v[0] = fmaf(at.weighed(u, e, d), d, v[0]);
        v[1] += w;
        v[2] = fmaf(w, d, v[2]);
      }
    if constexpr (BLOCK) {
      block_sums(v, s3);
    } else {
#pragma unroll
      for (int q = 0; q < 3; ++q) v[q] = group_sum<G>(v[q]);
    }
    const float rstd = rsqrt_of(n.mean(v[0]) + a.eps), mw = n.mean(v[1]), along = n.mean(v[2]) * rstd;
    if (!COLUMNS && sums && threadIdx.x == 0) reinterpret_cast<float2*>(sums)[row] = make_float2(mean, rstd);
    renew();
    Pack<T> out[U];
    if (BLOCK || row < a.rows) {
#pragma unroll
      for (int u = 0; u < U; ++u)
#pragma unroll
        for (int e = 0; e < V; ++e) {
          const float h = (float(x[u].v[e]) - mean) * rstd, y = float(dl[u].v[e]);
          out[u].v[e] = T(rstd * fmaf(-h, along, weighted(u, e) - mw));
          if constexpr (COLUMNS) {
            g_gain[u][e] = fmaf(y, h, g_gain[u][e]);
            g_bias[u][e] += y;
          }
        }
    }
    if (first + step < a.rows) load(row + step);  // before the stores, which it would wait for
    if (a.g_x && (BLOCK || row < a.rows)) {
      T* p = static_cast<T*>(a.g_x) + row * a.g_x_ld;
#pragma unroll
      for (int u = 0; u < U; ++u) at.store(p, u, out[u]);
    }
  }

  if constexpr (!COLUMNS) return;
  auto put = [&](int which, int64_t c, float t) {
    T* result = static_cast<T*>(which ? a.g_bias : a.g_gain);
    if (!result) return;
    if (gridDim.x == 1)
      result[c] = T(t);
    else
      sums[(int64_t(blockIdx.x) * 2 + which) * a.cols + c] = t;
  };
#pragma unroll
  for (int which = 0; which < 2; ++which)
#pragma unroll
    for (int u = 0; u < U; ++u) {
#pragma unroll
      for (int e = 0; e < V; ++e) {
        float t = which ? g_bias[COLUMNS ? u : 0][e] : g_gain[COLUMNS ? u : 0][e];
        if constexpr (BLOCK) {
          if (at.on(u) && at.counts(u, e)) put(which, at.at[u] + e, t);
        } else {
#pragma unroll
          for (int off = G; off < 64; off <<= 1) t += __shfl_xor(t, off);
          if (threadIdx.x % 64 < G) s_join[threadIdx.x / 64][lane * V + e] = t;
        }
      }
      if constexpr (!BLOCK) {
        __syncthreads();
        for (int c = threadIdx.x; c < G * V; c += THREADS) {
          const int col = u * G * V + c;  // packs that end with the row hold it further back
          const int l = c / V, shared = END == END_SHARED ? max(0, (u * G + l) * V - (int(a.cols) - V)) : 0;
          if (shared >= V) continue;
          const int e = c % V;
          const bool in = END == END_TINY ? e < a.cols : e >= shared;
          if (!in) continue;
          float t = s_join[0][c];
#pragma unroll
          for (int w = 1; w < WAVES; ++w) t += s_join[w][c];
          put(which, col - shared, t);
        }
        __syncthreads();
      }
    }
}

// ---- rows of any length: a block a row, read once for each sum -----------------
constexpr int kLongThreads = 1024, kLongWaves = kLongThreads / 64;
// f(first column, columns) of a thread's packs, four whole ones at a time as long as
// there are, so that four loads are on their way (with 256 threads and one at a time
// 1000 x 65536 f16 100 us, so 76; 64 x 1000003 f32 1511 and 478).  Bound by reading x
// again, out of the caches while all blocks' rows fit them.
template <typename T, typename F>
__device__ __forceinline__ void for_packs(int64_t cols, F&& f) {
  constexpr int N = Pack<T>::N, STEP = kLongThreads * N;
  int64_t c = int64_t(threadIdx.x) * N;
  for (; c + 3 * STEP + N <= cols; c += 4 * STEP) {
#pragma unroll
    for (int u = 0; u < 4; ++u) f(c + u * STEP, N);
  }
  for (; c < cols; c += STEP) f(c, int(min(int64_t(N), cols - c)));
}

template <typename T>
__device__ __forceinline__ float row_mean(const T* x, int64_t cols, float (&s)[kLongWaves][1]) {
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
__global__ __launch_bounds__(kLongThreads) void long_rows_kernel(const LayerNormArgs a) {
  __shared__ float s[kLongWaves][1];
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
__global__ __launch_bounds__(kLongThreads) void long_rows_grad_kernel(const LayerNormArgs a, float2* __restrict__ stats) {
  __shared__ float s1[kLongWaves][1], s3[kLongWaves][3];
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

// Sums over one part of the rows, for 64 packs of columns a block: sums[part] =
// [g_gain, g_bias], or, of all rows, the result.
template <typename T>
__global__ __launch_bounds__(kThreads) void column_grads_kernel(const LayerNormArgs a, const float2* __restrict__ stats,
                                                                int64_t part, float* __restrict__ sums) {
  constexpr int V = Pack<T>::N;
  __shared__ float s[kWaves][64 * V];
  const int lane = threadIdx.x % 64, wave = threadIdx.x / 64;
  const int64_t r0 = int64_t(blockIdx.x) * part, r1 = min(a.rows, r0 + part);
  for (int64_t j0 = int64_t(blockIdx.y) * 64 * V; j0 < a.cols; j0 += int64_t(gridDim.y) * 64 * V) {
    const int64_t j = j0 + lane * V;
    const int count = int(max(int64_t(0), min(int64_t(V), a.cols - j)));
    float gain[V] = {}, bias[V] = {};
    if (count > 0)
      for (int64_t r = r0 + wave; r < r1; r += kWaves) {
        const Pack<T> x = load_some(static_cast<const T*>(a.x) + r * a.x_ld + j, count);
        const Pack<T> dl = load_some(static_cast<const T*>(a.dl) + r * a.dl_ld + j, count);
        const float2 st = stats[r];
#pragma unroll
        for (int e = 0; e < V; ++e) {
          gain[e] = fmaf(float(dl.v[e]), (float(x.v[e]) - st.x) * st.y, gain[e]);
          bias[e] += float(dl.v[e]);
        }
      }
#pragma unroll
    for (int which = 0; which < 2; ++which) {
#pragma unroll
      for (int e = 0; e < V; ++e) s[wave][lane * V + e] = which ? bias[e] : gain[e];
      __syncthreads();
      for (int c = threadIdx.x; c < 64 * V; c += kThreads)
        if (j0 + c < a.cols) {
          const float t = (s[0][c] + s[1][c]) + (s[2][c] + s[3][c]);
          T* result = static_cast<T*>(which ? a.g_bias : a.g_gain);
          if (gridDim.x > 1)
            sums[(int64_t(blockIdx.x) * 2 + which) * a.cols + j0 + c] = t;
          else if (result)
            result[j0 + c] = T(t);
        }
      __syncthreads();
    }
  }
}

// g_gain and g_bias (either may be NULL) from the parts' sums: a block takes 16
// neighbouring sums, and its 64 groups of 16 lanes every 64th part.
constexpr int kJoinThreads = 1024, kJoinCols = 16, kJoinRows = kJoinThreads / kJoinCols;
template <typename T>
__global__ __launch_bounds__(kJoinThreads) void join_column_grads_kernel(const float* __restrict__ sums,
                                                                         int64_t parts, int64_t cols,
                                                                         T* __restrict__ g_gain,
                                                                         T* __restrict__ g_bias) {
  __shared__ float s[kJoinRows][kJoinCols + 1];
  const int c = threadIdx.x % kJoinCols, r = threadIdx.x / kJoinCols;
  for (int64_t b = int64_t(blockIdx.x) * kJoinCols; b < 2 * cols; b += int64_t(gridDim.x) * kJoinCols) {
    const int64_t e = b + c;
    T* to = e < cols ? g_gain : g_bias;
    float t = 0.0f;
    if (e < 2 * cols && to) {
#pragma unroll 8
      for (int64_t p = r; p < parts; p += kJoinRows) t += sums[p * 2 * cols + e];
    }
    s[r][c] = t;
    __syncthreads();
    static_assert(kJoinThreads / 64 == kJoinCols && kJoinRows == 64, "a wave a column");
    const int col = threadIdx.x / 64, at = threadIdx.x % 64;
    const float v = group_sum<64>(s[at][col]);
    const int64_t o = b + col;
    T* out = o < cols ? g_gain : g_bias;
    if (at == 0 && o < 2 * cols && out) out[o < cols ? o : o - cols] = T(v);
    __syncthreads();
  }
}

// f(integral constants G, U) for rows of `packs` packs: a wave's lanes up to 128 of
// them, with as few idle ones as two or three packs a lane allow (200000 x 130 f16,
// 17 packs: 30 us with 32 lanes, 22 with three packs in each of 8).
template <int N>
using Int = std::integral_constant<int, N>;
template <typename F>
void with_lanes(int64_t packs, F&& f) {
  if (packs <= 1) return f(Int<1>{}, Int<1>{});
  if (packs <= 2) return f(Int<2>{}, Int<1>{});
  if (packs <= 4) return f(Int<4>{}, Int<1>{});
  if (packs <= 8) return f(Int<8>{}, Int<1>{});
  if (packs <= 12) return f(Int<4>{}, Int<3>{});
  if (packs <= 16) return f(Int<16>{}, Int<1>{});
  if (packs <= 24) return f(Int<8>{}, Int<3>{});
  if (packs <= 32) return f(Int<32>{}, Int<1>{});
  if (packs <= 48) return f(Int<16>{}, Int<3>{});
  if (packs <= 64) return f(Int<64>{}, Int<1>{});
  if (packs <= 96) return f(Int<32>{}, Int<3>{});
  f(Int<64>{}, Int<2>{});
}
// f(threads, packs a thread) for longer rows, up to 4096 packs
template <typename F>
void with_block(int64_t packs, F&& f) {
  if (packs <= 256) return f(Int<256>{}, Int<1>{});
  if (packs <= 512) return f(Int<256>{}, Int<2>{});
  if (packs <= 1024) return f(Int<256>{}, Int<4>{});
  if (packs <= 2048) return f(Int<256>{}, Int<8>{});
  f(Int<512>{}, Int<8>{});
}
constexpr int64_t kWavePacks = 128, kBlockPacks = 4096;
constexpr int64_t kRowBlocks = 256 * 16;  // blocks that walk over the rows

template <typename T>
hipError_t forward(const LayerNormArgs& a, hipStream_t s) {
  if (a.rows <= 0 || a.cols <= 0) return hipSuccess;
  constexpr int V = Pack<T>::N;
  const int64_t packs = ceil_div64(a.cols, V);
  if (packs <= kWavePacks) {
    with_lanes(packs, [&](auto g, auto u) {
      constexpr int G = decltype(g)::value, U = decltype(u)::value;
      const uint32_t grid = uint32_t(std::min(ceil_div64(a.rows * G, kThreads), kRowBlocks));
      if (a.cols < V) {
        if constexpr (G == 1) rows_kernel<T, 1, 1, END_TINY><<<grid, kThreads, 0, s>>>(a);
      } else if (a.cols == G * U * V) {
        rows_kernel<T, G, U, END_EXACT><<<grid, kThreads, 0, s>>>(a);
      } else {
        rows_kernel<T, G, U, END_SHARED><<<grid, kThreads, 0, s>>>(a);
      }
    });
    return hipGetLastError();
  }
  if (packs <= kBlockPacks) {
    const uint32_t grid = uint32_t(std::min(a.rows, kMaxBlocks));
    with_block(packs, [&](auto t, auto u) {
      constexpr int THREADS = decltype(t)::value;
      block_rows_kernel<T, THREADS, decltype(u)::value><<<grid, THREADS, 0, s>>>(a);
    });
    return hipGetLastError();
  }
  long_rows_kernel<T><<<uint32_t(std::min(a.rows, kMaxBlocks)), kLongThreads, 0, s>>>(a);
  return hipGetLastError();
}

// The gradient's lanes and blocks: as many packs a lane as leave room for their column
// sums with four waves a SIMD (40000 x 700 f16, 88 packs: 54 us with two in each of 64
// lanes, 43 with three in 32; 9 to 12 packs lose by it, 200000 x 96 bf16 32 and 35).
constexpr int kGradThreads = 512;
template <typename F>
void with_grad_lanes(int64_t packs, F&& f) {
  if (packs <= 1) return f(Int<1>{}, Int<1>{});
  if (packs <= 2) return f(Int<2>{}, Int<1>{});
  if (packs <= 4) return f(Int<4>{}, Int<1>{});
  if (packs <= 8) return f(Int<8>{}, Int<1>{});
  if (packs <= 16) return f(Int<16>{}, Int<1>{});
  if (packs <= 24) return f(Int<8>{}, Int<3>{});
  if (packs <= 32) return f(Int<32>{}, Int<1>{});
  if (packs <= 48) return f(Int<16>{}, Int<3>{});
  if (packs <= 64) return f(Int<64>{}, Int<1>{});
  if (packs <= 96) return f(Int<32>{}, Int<3>{});
  f(Int<64>{}, Int<2>{});
}
// Longer rows, up to 8192 columns; past those the blocks would be one a CU.
constexpr int64_t kGradCols = 8192, kManyRows = 1024;
template <typename F>
void with_grad_block(int64_t packs, F&& f) {
  if (packs <= 256) return f(Int<256>{}, Int<1>{});
  if (packs <= 512) return f(Int<256>{}, Int<2>{});
  if (packs <= 1024) return f(Int<512>{}, Int<2>{});
  f(Int<1024>{}, Int<2>{});
}

struct Plan {
  bool fused;      // one kernel for rows and column sums
  int64_t parts;   // of the rows, that leave column sums
  int64_t part;    // rows of a part (not fused)
  size_t stats, total;
};
constexpr int64_t kFewColumnRows = 128, kPartRows = 16, kMaxParts = 2048, kCardPacks = 256 * 1024;
Plan plan_of(int64_t rows, int64_t cols, int64_t es) {
  Plan p{};
  const int64_t V = 16 / es, packs = ceil_div64(cols, V);
  // Rows of a block each are summed as they are read where there are many, a launch
  // later where their blocks would have few (64 x 16384 f16: 43 us, so 19; 64 x 4096
  // bf16 13.9 and 12.5).
  p.fused = packs <= kWavePacks || (cols <= kGradCols && rows >= kManyRows);
  if (p.fused) {
    int64_t at_once = 1, lanes = 0;  // rows a block takes at a time; its threads times their packs
    if (packs <= kWavePacks)
      with_grad_lanes(packs, [&](auto g, auto u) {
        at_once = kGradThreads / decltype(g)::value;
        lanes = kGradThreads * decltype(u)::value;
      });
    else
      with_grad_block(packs, [&](auto t, auto u) { lanes = decltype(t)::value * decltype(u)::value; });
    const int64_t turns = ceil_div64(rows, at_once);
    // A block alone spares the second launch.  Else parts as many as fill the card (twice
    // as many: 8191 x 4096 f16 65 us, so 60; half as many: 30000 x 2000 f16 101, so 86),
    // as long as their sums stay an eighth of the rows, or each has four turns left; and
    // all with as many turns.
    const int64_t most = std::min(std::max(rows * es / 43, turns / 4), std::max<int64_t>(256, kCardPacks / lanes));
    p.parts = turns <= 4 ? 1 : ceil_div64(turns, ceil_div64(turns, most));
    p.stats = p.parts > 1 ? size_t(ceil_div64(p.parts * 2 * cols * 4, 16)) * 16 : 0;
    p.total = p.stats;
    return p;
  }
  // Blocks of the column sums take all of few rows; else they fill the card.
  const int64_t across = ceil_div64(packs, 64);
  p.part = rows <= kFewColumnRows ? std::max<int64_t>(1, rows)
                                  : std::max(kPartRows, ceil_div64(rows, std::max<int64_t>(1, kMaxParts / across)));
  p.parts = ceil_div64(rows, p.part);
  p.stats = p.parts > 1 ? size_t(ceil_div64(p.parts * 2 * cols * 4, 16)) * 16 : 0;
  p.total = p.stats + size_t(rows) * sizeof(float2);
  return p;
}

template <typename T>
hipError_t rows_grad(const LayerNormArgs& a, const Plan& p, float* sums, hipStream_t s) {
  constexpr int V = Pack<T>::N;
  const int64_t packs = ceil_div64(a.cols, V);
  const uint32_t grid = uint32_t(p.parts);
  if (packs <= kWavePacks)
    with_grad_lanes(packs, [&](auto g, auto u) {
      constexpr int G = decltype(g)::value, U = decltype(u)::value;
      if (a.cols < V) {
        if constexpr (G == 1) rows_grad_kernel<T, 1, 1, END_TINY, kGradThreads, true><<<grid, kGradThreads, 0, s>>>(a, sums);
      } else if (a.cols == G * U * V) {
        rows_grad_kernel<T, G, U, END_EXACT, kGradThreads, true><<<grid, kGradThreads, 0, s>>>(a, sums);
      } else {
        rows_grad_kernel<T, G, U, END_SHARED, kGradThreads, true><<<grid, kGradThreads, 0, s>>>(a, sums);
      }
    });
  else
    with_grad_block(packs, [&](auto t, auto u) {
      constexpr int THREADS = decltype(t)::value;
      rows_grad_kernel<T, THREADS, decltype(u)::value, END_SHARED, THREADS, true><<<grid, THREADS, 0, s>>>(a, sums);
    });
  return hipGetLastError();
}

// g_x and the rows' mean and rstd.  Registers hold 16384 columns: with four 16-bit
// packs a lane 1024 threads would spill.
template <typename T>
constexpr int64_t kAlonePacks = sizeof(T) == 4 ? 4096 : 2048;
template <typename T>
hipError_t rows_alone(const LayerNormArgs& a, float2* stats, hipStream_t s) {
  const int64_t packs = ceil_div64(a.cols, Pack<T>::N);
  const uint32_t grid = uint32_t(std::min(a.rows, kMaxBlocks));
  auto launch = [&](auto t, auto u) {
    constexpr int THREADS = decltype(t)::value;
    rows_grad_kernel<T, THREADS, decltype(u)::value, END_SHARED, THREADS, false>
        <<<grid, THREADS, 0, s>>>(a, reinterpret_cast<float*>(stats));
  };
  if (packs <= 256)
    launch(Int<256>{}, Int<1>{});
  else if (packs <= 512)
    launch(Int<256>{}, Int<2>{});
  else if (packs <= 1024)
    launch(Int<512>{}, Int<2>{});
  else if (packs <= 2048)
    launch(Int<1024>{}, Int<2>{});
  else if (packs <= kAlonePacks<T>) {
    if constexpr (kAlonePacks<T> > 2048) launch(Int<1024>{}, Int<4>{});
  } else {
    long_rows_grad_kernel<T><<<grid, kLongThreads, 0, s>>>(a, stats);
  }
  return hipGetLastError();
}

template <typename T>
hipError_t backward(const LayerNormArgs& a, hipStream_t s) {
  if (a.cols <= 0) return hipSuccess;
  const Plan p = plan_of(a.rows, a.cols, sizeof(T));
  const bool columns = a.g_gain || a.g_bias;
  float* sums = static_cast<float*>(a.scratch);
  hipError_t e = hipSuccess;
  if (a.rows > 0 && (a.g_x || columns)) {
    if (p.fused) {
      if ((e = rows_grad<T>(a, p, sums, s)) != hipSuccess || p.parts == 1) return e;
    } else {
      float2* stats = reinterpret_cast<float2*>(static_cast<char*>(a.scratch) + p.stats);
      if ((e = rows_alone<T>(a, columns ? stats : nullptr, s)) != hipSuccess) return e;
      if (columns) {
        const dim3 parts(uint32_t(p.parts), uint32_t(std::min<int64_t>(ceil_div64(a.cols, 64 * Pack<T>::N), 65535)));
        column_grads_kernel<T><<<parts, kThreads, 0, s>>>(a, stats, p.part, sums);
        if ((e = hipGetLastError()) != hipSuccess || p.parts == 1) return e;
      }
    }
  }
  if (!columns) return e;
  const int64_t blocks = std::min<int64_t>(ceil_div64(2 * a.cols, kJoinCols), 1 << 16);
  join_column_grads_kernel<T><<<uint32_t(blocks), kJoinThreads, 0, s>>>(
      sums, a.rows > 0 ? p.parts : 0, a.cols, static_cast<T*>(a.g_gain), static_cast<T*>(a.g_bias));
  return hipGetLastError();
}

}  // namespace

size_t layer_norm_backward_scratch_bytes(int64_t rows, int64_t cols, gart_dtype t) {
  if (rows <= 0 || cols <= 0) return 0;
  return plan_of(rows, cols, int64_t(dtype_bytes(t))).total;
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
