// Orthogonalising a matrix by the products of a polynomial, and the momentum step
// that uses it.
//
//   X = x / (|x| + eps);  steps times:  A = X X^T,  P = b A + c A^2,  X <- a X + P X
//
// with X lying flat (the transpose of a tall x).  Each step moves every singular
// value s of X to a s + b s^3 + c s^5 and leaves the singular vectors.
//
// Products run on the float16 matrix cores with operands in two parts
// (orthogonalize.h): high high + high low + low high, sums in float, so that the
// result is float32's (2-norm 2.4e-6 off at 512 x 512, as the same steps in float32
// are).  With operands rounded once to float16 it is 1e-3 to 4e-3 off, more than
// bfloat16's rounding of the result.  Large float32 products run at 154 TFLOP/s on
// this card and float16 ones at 1430, so three of those are a third of the time.
// a X is added in float: inside P it would double the error.
#include "blocks.h"
#include "orthogonalize.h"
#include "tile.h"

namespace gart {
namespace {

constexpr int kThreads = 256;

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
  __device__ __forceinline__ float at(int64_t r, int64_t c) const {
    if (!m) return float(x[r * ld + c]);
    const float v = m[r * m_ld + c];
    return nesterov ? fmaf(momentum, v, float(x[r * ld + c])) : v;
  }
};

// m <- momentum m + g (if there is m), and the sum of squares of what is to be
// orthogonalised, in 64 bits: float's squares would overflow from 2e19 on.
template <typename T>
__global__ __launch_bounds__(kThreads) void squares_kernel(const Source<T> u, float* m, int64_t rows, int64_t cols,
                                                           double* __restrict__ sums) {
  __shared__ double s[kThreads / 64];
  const int lane = threadIdx.x % 64, wave = threadIdx.x / 64;
  double t = 0.0;
  for (int64_t r = int64_t(blockIdx.x) * (kThreads / 64) + wave; r < rows; r += int64_t(gridDim.x) * (kThreads / 64))
    for (int64_t c = lane; c < cols; c += 64) {
      if (m) m[r * u.m_ld + c] = fmaf(u.momentum, m[r * u.m_ld + c], float(u.x[r * u.ld + c]));
      const double v = double(u.at(r, c));
      t = fma(v, v, t);
    }
#pragma unroll
  for (int off = 32; off > 0; off >>= 1) t += __shfl_xor(t, off);
  if (lane == 0) s[wave] = t;
  __syncthreads();
  if (threadIdx.x == 0) sums[blockIdx.x] = (s[0] + s[1]) + (s[2] + s[3]);
}

// A float as high + low.
__device__ __forceinline__ void split(float v, f16& high, f16& low) {
  high = f16(v);
  low = f16(v - float(high));
}

// X in two parts, zero in the padding, from u over its norm: 64 x 64 elements a
// block; and the steps' factors, by the first one.
struct Iteration {
  float a, b, c, eps;
  int steps;
  Factors of_one;  // of values that start at 1
};
template <typename T>
__global__ __launch_bounds__(kThreads) void prepare_kernel(const Source<T> u, int64_t n, int64_t m, bool tall,
                                                           const double* __restrict__ sums, const Iteration it,
                                                           StepFactors* __restrict__ factors, f16* __restrict__ x,
                                                           int64_t x_ld, int64_t x_low) {
  __shared__ double s_sum[kThreads / 64];
  __shared__ float s_tile[64][65];
  const int lane = threadIdx.x % 64, wave = threadIdx.x / 64;
  static_assert(kSumBlocks == kThreads, "a partial sum a thread");
  double t = sums[threadIdx.x];
#pragma unroll
  for (int off = 32; off > 0; off >>= 1) t += __shfl_xor(t, off);
  if (lane == 0) s_sum[wave] = t;
  const int64_t i0 = int64_t(blockIdx.y) * 64, j0 = int64_t(blockIdx.x) * 64;
  for (int k = wave; k < 64; k += kThreads / 64) {
    // lanes along the source's columns
    const int i = tall ? lane : k, j = tall ? k : lane;
    float v = 0.0f;
    if (i0 + i < n && j0 + j < m) v = tall ? u.at(j0 + j, i0 + i) : u.at(i0 + i, j0 + j);
    s_tile[i][j] = v;
  }
  __syncthreads();
  const double size = sqrt((s_sum[0] + s_sum[1]) + (s_sum[2] + s_sum[3])), norm = size + double(it.eps);
  const bool tiny = size / norm < kNearOne;  // not if it is a NaN
  const double inv = (tiny ? pair_scale(size / norm, kMostX) : double(it.of_one.x)) / norm;
  if (blockIdx.x == 0 && blockIdx.y == 0) {
    if (!tiny) {
      if (threadIdx.x < it.steps) factors[threadIdx.x] = it.of_one.step[threadIdx.x];
    } else if (threadIdx.x == 0) {
      float first;
      step_factors(it.a, it.b, it.c, it.steps, size / norm, &first, factors);
    }
  }
  for (int c = threadIdx.x; c < 64 * 8; c += kThreads) {
    const int i = c / 8, j = c % 8 * 8;
    Pack<f16> high, low;
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      const bool in = i0 + i < n && j0 + j + e < m;
      const float v = in ? float(double(s_tile[i][j + e]) * inv) : 0.0f;  // padding stays 0 whatever the norm
      f16 h, l;
      split(v, h, l);
      high.v[e] = h;
      low.v[e] = l;
    }
    f16* to = x + (i0 + i) * x_ld + j0 + j;
    store_pack(to, high);
    store_pack(to + x_low, low);
  }
}

// ---- products of pairs ----------------------------------------------------------
enum PairEpilogue {
  PAIR_PAIR,  // the result in two parts
  PAIR_OUT,   // y
  PAIR_STEP   // param
};

// C = alpha sum_k A(i,k) B(j,k) + beta D(i,j).  All sizes are whole tiles.
struct PairArgs {
  const f16 *a, *b, *d;  // high parts; d may be NULL
  int64_t a_ld, b_ld, d_ld, a_low, b_low, d_low;
  int64_t tiles_i, tiles_j, depth;
  const float* factors;  // alpha, beta
  void* out;
  int64_t out_ld, out_low;  // PAIR_PAIR: elements to the low parts
  int64_t rows, cols;       // else: of out
  float decay, step;        // PAIR_STEP: param -= decay param + step C
};

// AKC, BKC: k runs along the operand's rows.  With A across k, D is read transposed.
template <typename T, bool AKC, bool BKC, int TI, int TJ, int WI, int WJ, PairEpilogue EPI>
__global__ __launch_bounds__(64 * WI * WJ) void pair_kernel(const PairArgs g) {
  using TA = Tile<f16, AKC, 16 * TI * WI, WI * WJ, false>;
  using TB = Tile<f16, BKC, 16 * TJ * WJ, WI * WJ, true>;
  constexpr int BI = 16 * TI * WI, BJ = 16 * TJ * WJ;
  constexpr int A_LOW = TA::ELEMS, B_HIGH = 2 * TA::ELEMS, B_LOW = B_HIGH + TB::ELEMS, ELEMS = B_LOW + TB::ELEMS;
  __shared__ __attribute__((aligned(16))) f16 lds[2][ELEMS];
  const int tid = threadIdx.x, lane = tid % 64, wave = __builtin_amdgcn_readfirstlane(tid / 64);
  const int wi = wave / WJ, wj = wave % WJ;
  const int64_t tile = xcd_tile(blockIdx.x, g.tiles_i * g.tiles_j);
  const int64_t i0 = tile / g.tiles_j * BI, j0 = tile % g.tiles_j * BJ;

  f32x4 acc[TI][TJ];
#pragma unroll
  for (int i = 0; i < TI; ++i)
#pragma unroll
    for (int j = 0; j < TJ; ++j) acc[i][j] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};

  TA ta;
  TB tb;
  ta.template aim<true>(g.a, g.a_ld, i0, g.tiles_i * BI, 0, tid);
  tb.template aim<true>(g.b, g.b_ld, j0, g.tiles_j * BJ, 0, tid);
  const int64_t a_step = TA::stride(g.a_ld), b_step = TB::stride(g.b_ld), steps = g.depth / kStep<f16>;
  auto fetch = [&](int h, int64_t n) {
    ta.fetch(lds[h], n * a_step, wave);
    ta.fetch(lds[h] + A_LOW, n * a_step + g.a_low, wave);
    tb.fetch(lds[h] + B_HIGH, n * b_step, wave);
    tb.fetch(lds[h] + B_LOW, n * b_step + g.b_low, wave);
  };
  fetch(0, 0);
  for (int64_t n = 0; n < steps; ++n) {
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");  // this wave's part of the buffer has landed
    __syncthreads();                                  // everyone's has, and the other buffer has been read
    if (n + 1 < steps) fetch((n + 1) & 1, n + 1);
    const f16* l = lds[n & 1];
#pragma unroll
    for (int s = 0; s < 2; ++s) {
      Pack<f16>::V ah[TI], al[TI], bh[TJ], bl[TJ];
#pragma unroll
      for (int i = 0; i < TI; ++i) {
        ah[i] = TA::fragment(l, wi * TI + i, s, lane);
        al[i] = TA::fragment(l + A_LOW, wi * TI + i, s, lane);
      }
#pragma unroll
      for (int j = 0; j < TJ; ++j) {
        bh[j] = TB::fragment(l + B_HIGH, wj * TJ + j, s, lane);
        bl[j] = TB::fragment(l + B_LOW, wj * TJ + j, s, lane);
      }
#pragma unroll
      for (int i = 0; i < TI; ++i)
#pragma unroll
        for (int j = 0; j < TJ; ++j) {
          acc[i][j] = Mfma<f16>::run(bl[j], ah[i], acc[i][j]);
          acc[i][j] = Mfma<f16>::run(bh[j], al[i], acc[i][j]);
          acc[i][j] = Mfma<f16>::run(bh[j], ah[i], acc[i][j]);
        }
    }
  }

  // A lane's columns: eight consecutive ones from each two tiles.
  const int r = lane % 16, q4 = lane / 16;
  const float alpha = g.factors[0], beta = g.factors[1];
#pragma unroll
  for (int jq = 0; jq < TJ / 2; ++jq) {
    const int64_t j = j0 + 32 * ((wj * TJ + jq * 2) / 2) + 8 * q4;
#pragma unroll
    for (int i = 0; i < TI; ++i) {
      const int64_t row = i0 + 16 * (wi * TI + i) + r;
      float c[8];
#pragma unroll
      for (int e = 0; e < 8; ++e) c[e] = alpha * acc[i][jq * 2 + e / 4][e % 4];
      if (g.d) {
        Pack<f16> dh, dl;
        if constexpr (AKC) {
          const f16* d = g.d + row * g.d_ld + j;
          dh = load_pack(d);
          dl = load_pack(d + g.d_low);
        } else {
#pragma unroll
          for (int e = 0; e < 8; ++e) {
            const f16* d = g.d + (j + e) * g.d_ld + row;
            dh.v[e] = d[0];
            dl.v[e] = d[g.d_low];
          }
        }
#pragma unroll
        for (int e = 0; e < 8; ++e) c[e] = fmaf(beta, float(dh.v[e]) + float(dl.v[e]), c[e]);
      }
      if constexpr (EPI == PAIR_PAIR) {
        Pack<f16> high, low;
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          f16 h, l;
          split(c[e], h, l);
          high.v[e] = h;
          low.v[e] = l;
        }
        f16* out = static_cast<f16*>(g.out) + row * g.out_ld + j;
        store_pack(out, high);
        store_pack(out + g.out_low, low);
      } else {
        if (row >= g.rows || j >= g.cols) continue;
        constexpr int V = Pack<T>::N;
        T* out = static_cast<T*>(g.out) + row * g.out_ld + j;
#pragma unroll
        for (int h = 0; h < 8 / V; ++h) {
          const int count = int(min(int64_t(V), g.cols - j - h * V));
          if (count <= 0) continue;
          Pack<T> p;
          if constexpr (EPI == PAIR_STEP) {
            p = load_some(out + h * V, count);
#pragma unroll
            for (int e = 0; e < V; ++e) {
              const float v = float(p.v[e]);
              p.v[e] = T(fmaf(-g.step, c[h * V + e], fmaf(-g.decay, v, v)));
            }
          } else {
#pragma unroll
            for (int e = 0; e < V; ++e) p.v[e] = T(c[h * V + e]);
          }
          store_some(out + h * V, p, count);
        }
      }
    }
  }
}

template <typename T, bool AKC, bool BKC, PairEpilogue EPI>
hipError_t run_pair(PairArgs g, int64_t rows, int64_t cols, hipStream_t s) {
  g.tiles_i = rows / 64;
  g.tiles_j = cols / 64;
  pair_kernel<T, AKC, BKC, 2, 2, 2, 2, EPI><<<uint32_t(g.tiles_i * g.tiles_j), 256, 0, s>>>(g);
  return hipGetLastError();
}

template <typename T>
hipError_t run(const OrthogonalizeArgs& a, hipStream_t s) {
  if (a.rows <= 0 || a.cols <= 0) return hipSuccess;
  const MatrixPlan p = matrix_plan(a.rows, a.cols);
  Iteration it{a.a, a.b, a.c, a.eps, a.steps, {}};
  if (!step_factors(a.a, a.b, a.c, a.steps, 1.0, &it.of_one.x, it.of_one.step)) return hipErrorInvalidValue;
  char* base = static_cast<char*>(a.scratch);
  double* sums = reinterpret_cast<double*>(base + p.sums);
  StepFactors* factors = reinterpret_cast<StepFactors*>(base + p.factors);
  f16* x[2] = {reinterpret_cast<f16*>(base + p.x[0]), reinterpret_cast<f16*>(base + p.x[1])};
  f16* gram = reinterpret_cast<f16*>(base + p.a);
  f16* poly = reinterpret_cast<f16*>(base + p.p);

  Source<T> u{static_cast<const T*>(a.x), a.x_ld, a.m, a.m_ld, a.momentum, a.nesterov};
  squares_kernel<T><<<uint32_t(kSumBlocks), kThreads, 0, s>>>(u, a.m, a.rows, a.cols, sums);
  hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;
  const dim3 grid(uint32_t(p.m_pad / 64), uint32_t(p.n_pad / 64));
  prepare_kernel<T><<<grid, kThreads, 0, s>>>(u, p.n, p.m, p.tall, sums, it, factors, x[0], p.m_pad, p.x_low);
  if ((e = hipGetLastError()) != hipSuccess) return e;

  for (int k = 0; k < a.steps; ++k) {
    PairArgs g{};
    g.a = g.b = x[k % 2];  // A = X X^T
    g.a_ld = g.b_ld = p.m_pad;
    g.a_low = g.b_low = p.x_low;
    g.depth = p.m_pad;
    g.factors = &factors[k].gram;
    g.out = gram;
    g.out_ld = p.n_pad;
    g.out_low = p.a_low;
    if ((e = run_pair<T, true, true, PAIR_PAIR>(g, p.n_pad, p.n_pad, s)) != hipSuccess) return e;
    g.a = g.b = g.d = gram;  // P = b A + c A A^T
    g.a_ld = g.b_ld = g.d_ld = p.n_pad;
    g.a_low = g.b_low = g.d_low = p.a_low;
    g.depth = p.n_pad;
    g.factors = &factors[k].square;
    g.out = poly;
    if ((e = run_pair<T, true, true, PAIR_PAIR>(g, p.n_pad, p.n_pad, s)) != hipSuccess) return e;
    const bool last = k + 1 == a.steps;
    g.a = poly;  // a X + P X
    g.b = g.d = x[k % 2];
    g.b_ld = g.d_ld = p.m_pad;
    g.b_low = g.d_low = p.x_low;
    g.factors = &factors[k].apply;
    if (!last) {
      g.out = x[(k + 1) % 2];
      g.out_ld = p.m_pad;
      g.out_low = p.x_low;
      e = run_pair<T, true, false, PAIR_PAIR>(g, p.n_pad, p.m_pad, s);
    } else {
      g.out = a.y;
      g.out_ld = a.y_ld;
      g.rows = a.rows;
      g.cols = a.cols;
      g.decay = a.decay;
      g.step = a.step;
      if (p.tall) {  // the transpose: rows of the result are columns of X
        std::swap(g.a, g.b);
        std::swap(g.a_ld, g.b_ld);
        std::swap(g.a_low, g.b_low);
        e = a.m ? run_pair<T, false, true, PAIR_STEP>(g, p.m_pad, p.n_pad, s)
                : run_pair<T, false, true, PAIR_OUT>(g, p.m_pad, p.n_pad, s);
      } else {
        e = a.m ? run_pair<T, true, false, PAIR_STEP>(g, p.n_pad, p.m_pad, s)
                : run_pair<T, true, false, PAIR_OUT>(g, p.n_pad, p.m_pad, s);
      }
    }
    if (e != hipSuccess) return e;
  }
  return e;
}

}  // namespace

int64_t orthogonalize_scratch_bytes(int64_t rows, int64_t cols) {
  if (rows <= 0 || cols <= 0) return 0;
  const MatrixPlan p = matrix_plan(rows, cols);
  if (p.n_pad / kTileSide > kMostTiles / (p.m_pad / kTileSide)) return -1;
  return int64_t(p.total);
}

hipError_t launch_orthogonalize(const OrthogonalizeArgs& a, gart_dtype t, hipStream_t s) {
  if (t == GART_DTYPE_F32) return run<float>(a, s);
  if (t == GART_DTYPE_BF16) return run<bf16>(a, s);
  return run<f16>(a, s);
}

}  // namespace gart
