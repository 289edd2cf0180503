// A small matrix through all its steps in one block: the step of a 48 x 64 f32 weight
// in 15 us, where 17 launches take 60.
//
// X stays in registers, as floats, TX tiles a wave; LDS holds its
// transpose in blocks and, one after the other, X itself, A and P.  What a wave adds
// to its sums it has in registers: A's tile to P's, X's to the next X's.  Bound by the
// chain of phases: each waits for LDS reads, a few dependent matrix instructions and
// a barrier.
#pragma once

#include "orthogonalize_device.h"

namespace gart {
namespace {

constexpr int kSmallWaves = 16, kSmallThreads = 64 * kSmallWaves;
constexpr int64_t kSmallElements = 19456;  // of the matrix padded to 32, up to 64 x 288, say: two of them in LDS
constexpr int64_t kSmallSide = 128;        // of A, which is one tile a wave at most

inline int64_t pad32(int64_t v) { return (v + 31) / 32 * 32; }
inline bool small_fits(const MatrixPlan& p) {
  return pad32(p.n) <= kSmallSide && pad32(p.n) * pad32(p.m) <= kSmallElements;
}

// sum over k of A(i,k) B(j,k): FRAG x FRAG fragments from row tiles ti and tj
template <int FRAG>
__device__ __forceinline__ void small_product(f32x4 (&sum)[FRAG][FRAG], const Blocks& a, const Blocks& b, int ti, int tj,
                                              int steps, int lane) {
#pragma unroll
  for (int i = 0; i < FRAG; ++i)
#pragma unroll
    for (int j = 0; j < FRAG; ++j) sum[i][j] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll(FRAG == 1 ? 2 : 1)
  for (int k = 0; k < steps; ++k) {
    Pack<f16>::V ah[FRAG], al[FRAG], bh[FRAG], bl[FRAG];
#pragma unroll
    for (int i = 0; i < FRAG; ++i) {
      const f16* p = a.at(ti * FRAG + i, k) + lane * 8;
      const f16* q = b.at(tj * FRAG + i, k) + lane * 8;
      ah[i] = *reinterpret_cast<const Pack<f16>::V*>(p);
      al[i] = *reinterpret_cast<const Pack<f16>::V*>(p + Blocks::kBlock);
      bh[i] = *reinterpret_cast<const Pack<f16>::V*>(q);
      bl[i] = *reinterpret_cast<const Pack<f16>::V*>(q + Blocks::kBlock);
    }
#pragma unroll
    for (int p = 0; p < 3; ++p)
#pragma unroll
      for (int i = 0; i < FRAG; ++i)
#pragma unroll
        for (int j = 0; j < FRAG; ++j)
          sum[i][j] = Mfma<f16>::run(p == 0 ? bl[j] : bh[j], p == 1 ? al[i] : ah[i], sum[i][j]);
  }
#pragma unroll
  for (int i = 0; i < FRAG; ++i)
#pragma unroll
    for (int j = 0; j < FRAG; ++j) arrive(sum[i][j]);  // read before the barrier behind which LDS is written again
}

// Four consecutive columns of a row into blocks, and into those of the transpose.
__device__ __forceinline__ void put_row(const Blocks& to, int row, int col, const f32x4& v) {
  typedef f16 f16x4 __attribute__((ext_vector_type(4)));
  f16x4 high, low;
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    f16 h, l;
    split(v[e], h, l);
    high[e] = h;
    low[e] = l;
  }
  f16* p = to.at(row / 16, col / 32) + (col % 32 / 8 * 16 + row % 16) * 8 + col % 8;
  *reinterpret_cast<f16x4*>(p) = high;
  *reinterpret_cast<f16x4*>(p + Blocks::kBlock) = low;
}
__device__ __forceinline__ void put_column(const Blocks& to, int row, int col, const f32x4& v) {
  f16* p = to.at(col / 16, row / 32) + (row % 32 / 8 * 16 + col % 16) * 8 + row % 8;
#pragma unroll
  for (int e = 0; e < 4; ++e) {  // col is a multiple of 4: four rows of one block
    f16 h, l;
    split(v[e], h, l);
    p[8 * e] = h;
    p[8 * e + Blocks::kBlock] = l;
  }
}

// The four elements from (i, j) of X in x, or in its transpose; 0 past the first `count`.
template <typename T>
struct __attribute__((packed)) Four {
  T v[4];
};
template <typename T>
__device__ __forceinline__ f32x4 load_four(const T* x, int64_t ld, bool tall, int i, int j, int count) {
  f32x4 r = {0.0f, 0.0f, 0.0f, 0.0f};
  if (!tall && count == 4) {
    const Four<T> f = *reinterpret_cast<const Four<T>*>(x + i * ld + j);
#pragma unroll
    for (int e = 0; e < 4; ++e) r[e] = float(f.v[e]);
  } else {
    const T* p = tall ? x + j * ld + i : x + i * ld + j;
    const int64_t step = tall ? ld : 1;
#pragma unroll
    for (int e = 0; e < 4; ++e)
      if (e < count) r[e] = float(p[e * step]);
  }
  return r;
}
template <typename T>
__device__ __forceinline__ void store_four(T* x, int64_t ld, bool tall, int i, int j, int count, const f32x4& r) {
  if (!tall && count == 4) {
    Four<T> f;
#pragma unroll
    for (int e = 0; e < 4; ++e) f.v[e] = T(r[e]);
    *reinterpret_cast<Four<T>*>(x + i * ld + j) = f;
  } else {
    T* p = tall ? x + j * ld + i : x + i * ld + j;
    const int64_t step = tall ? ld : 1;
#pragma unroll
    for (int e = 0; e < 4; ++e)
      if (e < count) p[e * step] = T(r[e]);
  }
}

// 16 waves, with a tile of A and TX of X each at most.  <T, 2, 2> spills 7 or 8
// registers: 128 x 128 f32 49 us (128 x 129, past what it takes, 65).
template <typename T, int FRAG, int TX>
__global__ __launch_bounds__(kSmallThreads) void small_kernel(const Source<T> u, float* m, int64_t rows, int64_t cols,
                                                              bool tall, const Iteration it, T* y, int64_t y_ld,
                                                              float decay, float step) {
  __shared__ __attribute__((aligned(16))) f16 s_xt[2 * kSmallElements], s_x[2 * kSmallElements];
  __shared__ StepFactors s_factors[kMaxSteps];
  __shared__ double s_sum[kSmallWaves];
  constexpr int SIDE = 16 * FRAG;
  const int lane = threadIdx.x % 64, wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64);
  const int r = lane % 16, g4 = lane / 16;
  const int n = int(tall ? cols : rows), k = int(tall ? rows : cols);  // X is n x k
  const int n_pad = (n + 31) / 32 * 32, k_pad = (k + 31) / 32 * 32;
  const int down = n_pad / SIDE, along = k_pad / SIDE;
  const Blocks x{s_x, k_pad / 32}, xt{s_xt, n_pad / 32}, a{s_x, n_pad / 32};  // P takes A's place

  // Each element is one lane's from beginning to end: of tile t, row i and columns j .. j + 3 of X.
  auto where = [&](int t, int p, int q, int& i, int& j) {
    const int tile = wave + t * kSmallWaves;
    i = tile / along * SIDE + 16 * p + r;
    j = tile % along * SIDE + 16 * q + 4 * g4;
    return tile < down * along;
  };
  // f(p, q, i, j, how many of the four elements from (i, j) of X there are) in tile t
  auto each = [&](int t, auto&& f) {
#pragma unroll
    for (int p = 0; p < FRAG; ++p)
#pragma unroll
      for (int q = 0; q < FRAG; ++q) {
        int i, j;
        const bool any = where(t, p, q, i, j);
        f(p, q, i, j, any && i < n ? max(0, min(4, k - j)) : 0);
      }
  };
  // A tile's loads are asked for before its first store, which they could not pass;
  // the parameters at the start, if there are registers for them.
  constexpr bool EARLY = FRAG == 1;
  f32x4 v[TX][FRAG][FRAG], old[FRAG][FRAG], param[EARLY ? TX : 1][FRAG][FRAG];
  auto load_param = [&](int t) {
    each(t, [&](int p, int q, int i, int j, int count) {
      param[EARLY ? t : 0][p][q] = load_four(y, y_ld, tall, i, j, count);
    });
  };
#pragma unroll
  for (int t = 0; t < TX; ++t) {
    each(t, [&](int p, int q, int i, int j, int count) { v[t][p][q] = load_four(u.x, u.ld, tall, i, j, count); });
    if (!m) continue;
    each(t, [&](int p, int q, int i, int j, int count) { old[p][q] = load_four(m, u.m_ld, tall, i, j, count); });
    if (EARLY) load_param(t);
    each(t, [&](int p, int q, int i, int j, int count) {
      f32x4 next;
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const float g = v[t][p][q][e];
        next[e] = fmaf(u.momentum, old[p][q][e], g);
        v[t][p][q][e] = u.nesterov ? fmaf(u.momentum, next[e], g) : next[e];  // 0 where there is nothing
      }
      store_four(m, u.m_ld, tall, i, j, count, next);
    });
  }
  double square = 0.0;
#pragma unroll
  for (int t = 0; t < TX; ++t)
#pragma unroll
    for (int p = 0; p < FRAG; ++p)
#pragma unroll
      for (int q = 0; q < FRAG; ++q)
#pragma unroll
        for (int e = 0; e < 4; ++e) square = fma(double(v[t][p][q][e]), double(v[t][p][q][e]), square);
#pragma unroll
  for (int off = 32; off > 0; off >>= 1) square += __shfl_xor(square, off);
  if (lane == 0) s_sum[wave] = square;
  if (threadIdx.x < it.steps) s_factors[threadIdx.x] = it.of_one.step[threadIdx.x];
  __syncthreads();
  square = 0.0;
#pragma unroll
  for (int w = 0; w < kSmallWaves; ++w) square += s_sum[w];
  const double size = sqrt(square);
  bool tiny;
  const double inv = first_scale(it, size, tiny);
  if (tiny) {
    __syncthreads();
    if (threadIdx.x == 0) {
      float first;
      step_factors(it.a, it.b, it.c, it.steps, size / (size + double(it.eps)), &first, s_factors);
    }
  }
  auto place = [&]() {
#pragma unroll
    for (int t = 0; t < TX; ++t)
#pragma unroll
      for (int p = 0; p < FRAG; ++p)
#pragma unroll
        for (int q = 0; q < FRAG; ++q) {
          int i, j;
          if (!where(t, p, q, i, j)) continue;
          put_row(x, i, j, v[t][p][q]);
          put_column(xt, i, j, v[t][p][q]);
        }
  };
#pragma unroll
  for (int t = 0; t < TX; ++t)
#pragma unroll
    for (int p = 0; p < FRAG; ++p)
#pragma unroll
      for (int q = 0; q < FRAG; ++q) {
        int i, j;
        const bool any = where(t, p, q, i, j);
#pragma unroll
        for (int e = 0; e < 4; ++e)  // padding stays 0 whatever the norm
          v[t][p][q][e] = any && i < n && j + e < k ? float(double(v[t][p][q][e]) * inv) : 0.0f;
      }
  place();
  __syncthreads();

  const int ai = wave / down, aj = wave % down;  // this wave's tile of A
  const bool has_a = wave < down * down;
  f32x4 gram[FRAG][FRAG];
  auto put_a = [&]() {
    __syncthreads();  // what lies there has been read
    if (has_a) {
#pragma unroll
      for (int p = 0; p < FRAG; ++p)
#pragma unroll
        for (int q = 0; q < FRAG; ++q) put_row(a, ai * SIDE + 16 * p + r, aj * SIDE + 16 * q + 4 * g4, gram[p][q]);
    }
    __syncthreads();
  };
  for (int s = 0; s < it.steps; ++s) {
    const StepFactors f = s_factors[s];
    f32x4 sum[FRAG][FRAG];
    if (has_a) {  // A = X X^T
      small_product<FRAG>(sum, x, x, ai, aj, k_pad / 32, lane);
#pragma unroll
      for (int p = 0; p < FRAG; ++p)
#pragma unroll
        for (int q = 0; q < FRAG; ++q) gram[p][q] = f.gram * sum[p][q];
    }
    put_a();
    if (has_a) {  // P = b A + c A A
      small_product<FRAG>(sum, a, a, ai, aj, n_pad / 32, lane);
#pragma unroll
      for (int p = 0; p < FRAG; ++p)
#pragma unroll
        for (int q = 0; q < FRAG; ++q)
#pragma unroll
          for (int e = 0; e < 4; ++e) gram[p][q][e] = fmaf(f.linear, gram[p][q][e], f.square * sum[p][q][e]);
    }
    put_a();
#pragma unroll
    for (int t = 0; t < TX; ++t) {  // a X + P X
      const int tile = wave + t * kSmallWaves;
      if (tile >= down * along) continue;
      small_product<FRAG>(sum, a, xt, tile / along, tile % along, n_pad / 32, lane);
#pragma unroll
      for (int p = 0; p < FRAG; ++p)
#pragma unroll
        for (int q = 0; q < FRAG; ++q)
#pragma unroll
          for (int e = 0; e < 4; ++e) v[t][p][q][e] = fmaf(f.keep, v[t][p][q][e], f.apply * sum[p][q][e]);
    }
    if (s + 1 < it.steps) {
      __syncthreads();
      place();
      __syncthreads();
    }
  }

#pragma unroll
  for (int t = 0; t < TX; ++t) {
    if (m) {
      if (!EARLY) load_param(t);
      each(t, [&](int p, int q, int, int, int) {
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const float w = param[EARLY ? t : 0][p][q][e];
          v[t][p][q][e] = fmaf(-step, v[t][p][q][e], fmaf(-decay, w, w));
        }
      });
    }
    each(t, [&](int p, int q, int i, int j, int count) { store_four(y, y_ld, tall, i, j, count, v[t][p][q]); });
  }
}

template <typename T>
hipError_t run_small(const OrthogonalizeArgs& a, const MatrixPlan& p, const Iteration& it, hipStream_t s) {
  Source<T> u{static_cast<const T*>(a.x), a.x_ld, a.m, a.m_ld, a.momentum, a.nesterov};
  T* y = static_cast<T*>(a.y);
  auto launch = [&](auto kernel) {
    kernel<<<1, kSmallThreads, 0, s>>>(u, a.m, a.rows, a.cols, p.tall, it, y, a.y_ld, a.decay, a.step);
  };
  const int64_t n = pad32(p.n), elements = n * pad32(p.m);
  // tiles of 16 where the waves suffice for them: half as many of 32 leave most waves
  // idle (48 x 64 f32 with four waves: 27 us, so 15)
  if (n <= 64 && elements <= kSmallWaves * 256)
    launch(small_kernel<T, 1, 1>);
  else if (n <= 64 && elements <= 2 * kSmallWaves * 256)
    launch(small_kernel<T, 1, 2>);
  else
    launch(small_kernel<T, 2, 2>);
  return hipGetLastError();
}

}  // namespace
}  // namespace gart
