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

// Of a 64 x 64 tile in LDS, element (i, j) at tile[i * pitch + j], into blocks: those
// of rows i, or, transposed, of rows j.  Values are split into two parts.
constexpr int kTilePitch = 64 + 4;
template <bool TRANSPOSED>
__device__ __forceinline__ void store_blocks(const float* tile, const Blocks& to, int64_t row0, int64_t col0, int lane,
                                             int first, int step) {
  const int r = lane % 16, g = lane / 16;
  for (int b = first; b < 8; b += step) {
    const int row = 16 * (b / 2) + r, k = 32 * (b % 2) + 8 * g;
    Pack<f16> high, low;
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      f16 h, l;
      split(TRANSPOSED ? tile[(k + e) * kTilePitch + row] : tile[row * kTilePitch + k + e], h, l);
      high.v[e] = h;
      low.v[e] = l;
    }
    f16* block = to.at(row0 / 16 + b / 2, col0 / 32 + b % 2) + lane * 8;
    store_pack(block, high);
    store_pack(block + Blocks::kBlock, low);
  }
}

// X and its transpose, zero in the padding, from u over its norm: 64 x 64 elements a
// block; and the steps' factors, by the first one.
struct Iteration {
  float a, b, c, eps;
  int steps;
  Factors of_one;  // of values that start at 1
};
template <typename T>
__global__ __launch_bounds__(kThreads) void prepare_kernel(const Source<T> u, int64_t n, int64_t m, bool tall,
                                                           const double* __restrict__ sums, const Iteration it,
                                                           StepFactors* __restrict__ factors, const Blocks x,
                                                           const Blocks xt) {
  __shared__ double s_sum[kThreads / 64];
  __shared__ float s_tile[64 * kTilePitch];
  const int lane = threadIdx.x % 64, wave = threadIdx.x / 64;
  static_assert(kSumBlocks == kThreads, "a partial sum a thread");
  double t = sums[threadIdx.x];
#pragma unroll
  for (int off = 32; off > 0; off >>= 1) t += __shfl_xor(t, off);
  if (lane == 0) s_sum[wave] = t;
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
  const int64_t i0 = int64_t(blockIdx.y) * 64, j0 = int64_t(blockIdx.x) * 64;
  for (int k = wave; k < 64; k += kThreads / 64) {
    // lanes along the source's columns
    const int i = tall ? lane : k, j = tall ? k : lane;
    float v = 0.0f;  // the padding stays 0 whatever the norm
    if (i0 + i < n && j0 + j < m) v = float(double(tall ? u.at(j0 + j, i0 + i) : u.at(i0 + i, j0 + j)) * inv);
    s_tile[i * kTilePitch + j] = v;
  }
  __syncthreads();
  store_blocks<false>(s_tile, x, i0, j0, lane, wave, kThreads / 64);
  store_blocks<true>(s_tile, xt, j0, i0, lane, wave, kThreads / 64);
}

// ---- products of pairs ----------------------------------------------------------
enum PairEpilogue {
  PAIR_BLOCKS,  // the result in blocks, and its transpose
  PAIR_OUT,     // y
  PAIR_STEP,    // param
  PAIR_PART     // float sums of one part of k
};

// C = alpha sum_k A(i,k) B(j,k) + beta D(i,j).  Sizes are multiples of 64, of zeros
// where the matrix ends.
struct PairArgs {
  Blocks a, b, d;       // d.data may be NULL
  int64_t rows, cols;   // of C
  int64_t steps;        // blocks along k
  int tiles_i, tiles_j, band;
  bool symmetric;       // C is: tiles above the diagonal are stored on both sides of it
  int parts;            // of k: blockIdx.y
  float* partial;       // their sums
  const float* factors; // alpha, beta
  Blocks out, across;   // PAIR_BLOCKS: C and, unless it is symmetric, its transpose
  void* y;              // else: the result
  int64_t y_ld, y_rows, y_cols;
  float decay, step;    // PAIR_STEP: y -= decay y + step C
};

// Blocks go to the eight XCDs in turn.  Each gets a run of tiles that covers a patch
// of `band` rows, so that its cache takes in few rows of both operands.  A triangle of
// tiles (i <= j) is folded to half as many rows: row r, then row n - 1 - r.
__device__ __forceinline__ bool find_tile(const PairArgs& g, int b, int total, int& ti, int& tj) {
  const int t = int(xcd_tile(b, total));
  const int n = g.tiles_i, even = n + n % 2;
  const int rows = g.symmetric ? even / 2 : n, cols = g.symmetric ? even + 1 : g.tiles_j;
  const int top = t / (g.band * cols) * g.band, high = min(g.band, rows - top);
  const int in = t - top * cols, r = top + in % high, c = in / high;
  ti = r;
  tj = c;
  if (g.symmetric) {
    const bool folded = c >= even - r;
    ti = folded ? even - 1 - r : r;
    tj = folded ? ti + c - (even - r) : r + c;
  }
  return ti < n && tj < g.tiles_j;
}

// A wave has 64 x 64 elements: WI x WJ waves a block, and WK of them take every WK-th
// block of k.  Two fragments' loads are on their way while one set is multiplied: the
// waves meet only when their sums are joined, in LDS.  JOIN: the sums of k are those
// of g.parts parts.
constexpr int kSide = 64, kFrag = 4;  // 16-row tiles a wave's side
template <typename T, int WI, int WJ, int WK, PairEpilogue EPI, bool JOIN>
__global__ __launch_bounds__(64 * WI * WJ * WK, 1) void pair_kernel(const PairArgs g) {
  constexpr int WAVES = WI * WJ * WK, THREADS = 64 * WAVES;
  constexpr int ROWS = kFrag / WK;  // 16-row tiles of a wave's result
  static_assert(WK == 1 || (WI == 1 && WJ == 1 && WK == kFrag), "one tile, or waves that share nothing");
  // joined sums, then tiles that are transposed
  __shared__ __attribute__((aligned(16))) float lds[WK > 1 && !JOIN ? WK * kSide * kSide
                                                    : EPI == PAIR_BLOCKS ? WI * WJ * kSide * kTilePitch : 4];
  const int tid = threadIdx.x, lane = tid % 64, wave = __builtin_amdgcn_readfirstlane(tid / 64);
  const int wk = wave % WK, wi = wave / WK / WJ, wj = wave / WK % WJ;
  int ti, tj;
  if (!find_tile(g, blockIdx.x, gridDim.x, ti, tj)) return;
  const int64_t i0 = (int64_t(ti) * WI + wi) * kSide, j0 = (int64_t(tj) * WJ + wj) * kSide;
  const bool inside = i0 < g.rows && j0 < g.cols;

  f32x4 acc[ROWS][kFrag];
  if constexpr (JOIN) {
#pragma unroll
    for (int i = 0; i < ROWS; ++i)
#pragma unroll
      for (int j = 0; j < kFrag; ++j) acc[i][j] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
    for (int part = 0; part < g.parts; ++part) {
      const float* from = g.partial + (int64_t(part) * gridDim.x + blockIdx.x) * (THREADS * ROWS * kFrag * 4) + tid * 4;
#pragma unroll
      for (int i = 0; i < ROWS; ++i)
#pragma unroll
        for (int j = 0; j < kFrag; ++j)
          acc[i][j] += *reinterpret_cast<const f32x4*>(from + (i * kFrag + j) * THREADS * 4);
    }
  } else {
    f32x4 sum[kFrag][kFrag];
#pragma unroll
    for (int i = 0; i < kFrag; ++i)
#pragma unroll
      for (int j = 0; j < kFrag; ++j) sum[i][j] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
    const int part = EPI == PAIR_PART ? int(blockIdx.y) : 0, parts = EPI == PAIR_PART ? g.parts : 1;
    const int k0 = int(g.steps * part / parts) + wk, k1 = int(g.steps * (part + 1) / parts);
    if (inside && k0 < k1) {
      const int64_t a_row = g.a.across * Blocks::kPair, b_row = g.b.across * Blocks::kPair;
      const f16* a = g.a.at(i0 / 16, k0) + lane * 8;
      const f16* b = g.b.at(j0 / 16, k0) + lane * 8;
      struct Set {
        Pack<f16>::V ah[kFrag], al[kFrag], bh[kFrag], bl[kFrag];
      } set[3];
      auto load = [&](Set& f, int n) {  // past the end the last one again
        const int64_t at = int64_t(min(n, (k1 - 1 - k0) / WK)) * (WK * Blocks::kPair);
#pragma unroll
        for (int i = 0; i < kFrag; ++i) {
          f.ah[i] = *reinterpret_cast<const Pack<f16>::V*>(a + i * a_row + at);
          f.al[i] = *reinterpret_cast<const Pack<f16>::V*>(a + i * a_row + at + Blocks::kBlock);
          f.bh[i] = *reinterpret_cast<const Pack<f16>::V*>(b + i * b_row + at);
          f.bl[i] = *reinterpret_cast<const Pack<f16>::V*>(b + i * b_row + at + Blocks::kBlock);
        }
        __builtin_amdgcn_sched_barrier(0);  // loads are asked for here, not where they are used
      };
      auto multiply = [&](const Set& f) {
#pragma unroll
        for (int p = 0; p < 3; ++p)
#pragma unroll
          for (int i = 0; i < kFrag; ++i)
#pragma unroll
            for (int j = 0; j < kFrag; ++j)
              sum[i][j] = Mfma<f16>::run(p == 0 ? f.bl[j] : f.bh[j], p == 1 ? f.al[i] : f.ah[i], sum[i][j]);
        __builtin_amdgcn_sched_barrier(0);
      };
      const int count = (k1 - k0 + WK - 1) / WK;
      load(set[0], 0);
      load(set[1], 1);
      int n = 0;
      for (; n + 2 < count; n += 3) {
        load(set[2], n + 2);
        multiply(set[0]);
        load(set[0], n + 3);
        multiply(set[1]);
        load(set[1], n + 4);
        multiply(set[2]);
      }
      if (n < count) multiply(set[0]);
      if (n + 1 < count) multiply(set[1]);
    }
    if constexpr (WK == 1) {
#pragma unroll
      for (int i = 0; i < kFrag; ++i)
#pragma unroll
        for (int j = 0; j < kFrag; ++j) acc[i][j] = sum[i][j];
    } else {
      // wave w takes the 16-row tile w of the others
#pragma unroll
      for (int i = 0; i < kFrag; ++i)
#pragma unroll
        for (int j = 0; j < kFrag; ++j)
          *reinterpret_cast<f32x4*>(lds + ((wave * kFrag + i) * kFrag + j) * 256 + lane * 4) = sum[i][j];
      __syncthreads();
#pragma unroll
      for (int j = 0; j < kFrag; ++j) {
        acc[0][j] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
        for (int w = 0; w < WK; ++w)
          acc[0][j] += *reinterpret_cast<const f32x4*>(lds + ((w * kFrag + wave) * kFrag + j) * 256 + lane * 4);
      }
      __syncthreads();
    }
  }

  if constexpr (EPI == PAIR_PART) {
    float* to = g.partial + (int64_t(blockIdx.y) * gridDim.x + blockIdx.x) * (THREADS * ROWS * kFrag * 4) + tid * 4;
#pragma unroll
    for (int i = 0; i < ROWS; ++i)
#pragma unroll
      for (int j = 0; j < kFrag; ++j) *reinterpret_cast<f32x4*>(to + (i * kFrag + j) * THREADS * 4) = acc[i][j];
    return;
  }

  // The fragments of B are not paired up: a lane has four consecutive columns of a row.
  const int r = lane % 16, g4 = lane / 16;
  const float alpha = g.factors[0], beta = g.factors[1];
  float* tile = lds + (WK > 1 ? 0 : wave * kSide * kTilePitch);
  if (inside) {
#pragma unroll
    for (int i = 0; i < ROWS; ++i) {
      const int row = 16 * (WK > 1 ? wave : i) + r;
#pragma unroll
      for (int j = 0; j < kFrag; ++j) {
        const int col = 16 * j + 4 * g4;
        f32x4 c = alpha * acc[i][j];
        if (g.d.data) {
          typedef f16 f16x4 __attribute__((ext_vector_type(4)));
          const f16* d = g.d.at((i0 + row) / 16, (j0 + col) / 32) + ((col % 32) / 8 * 16 + r) * 8 + col % 8;
          const f16x4 dh = *reinterpret_cast<const f16x4*>(d), dl = *reinterpret_cast<const f16x4*>(d + Blocks::kBlock);
#pragma unroll
          for (int e = 0; e < 4; ++e) c[e] = fmaf(beta, float(dh[e]) + float(dl[e]), c[e]);
        }
        if constexpr (EPI == PAIR_BLOCKS) {
          *reinterpret_cast<f32x4*>(tile + row * kTilePitch + col) = c;
        } else {
          if (i0 + row >= g.y_rows || j0 + col >= g.y_cols) continue;
          T* y = static_cast<T*>(g.y) + (i0 + row) * g.y_ld + j0 + col;
          const int count = int(min(int64_t(4), g.y_cols - j0 - col));
          struct __attribute__((packed)) Four {
            T v[4];
          };
          Four f;
          auto each = [&](int e, T& v) {
            if constexpr (EPI == PAIR_STEP) {
              const float p = float(v);
              v = T(fmaf(-g.step, c[e], fmaf(-g.decay, p, p)));
            } else {
              v = T(c[e]);
            }
          };
          if (count == 4) {
            if constexpr (EPI == PAIR_STEP) f = *reinterpret_cast<const Four*>(y);
#pragma unroll
            for (int e = 0; e < 4; ++e) each(e, f.v[e]);
            *reinterpret_cast<Four*>(y) = f;
          } else {
#pragma unroll
            for (int e = 0; e < 4; ++e)
              if (e < count) each(e, y[e]);
          }
        }
      }
    }
  }
  if constexpr (EPI == PAIR_BLOCKS) {
    __syncthreads();
    if (!inside) return;
    constexpr int SHARE = WK;  // waves that store the tile
    store_blocks<false>(tile, g.out, i0, j0, lane, wk, SHARE);
    if (g.symmetric) {
      if (i0 != j0) store_blocks<true>(tile, g.out, j0, i0, lane, wk, SHARE);
    } else {
      store_blocks<true>(tile, g.across, j0, i0, lane, wk, SHARE);
    }
  }
}

template <typename T, int W, int WK, PairEpilogue EPI>
hipError_t run_tiles(PairArgs g, const PairCut& c, hipStream_t s) {
  g.tiles_i = int((g.rows + c.side - 1) / c.side);
  g.tiles_j = int((g.cols + c.side - 1) / c.side);
  g.symmetric = c.symmetric;
  g.parts = c.parts;
  const uint32_t blocks = uint32_t(blocks_of(g.rows, g.cols, c.side, c.symmetric));
  g.band = 1;
  while (g.band * g.band * 8 < int(blocks)) ++g.band;
  constexpr int THREADS = 64 * W * W * WK;
  if (c.parts == 1) {
    pair_kernel<T, W, W, WK, EPI, false><<<blocks, THREADS, 0, s>>>(g);
    return hipGetLastError();
  }
  if constexpr (EPI == PAIR_BLOCKS) {
    pair_kernel<T, W, W, WK, PAIR_PART, false><<<dim3(blocks, uint32_t(c.parts)), THREADS, 0, s>>>(g);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
    pair_kernel<T, W, W, WK, PAIR_BLOCKS, true><<<blocks, THREADS, 0, s>>>(g);
    return hipGetLastError();
  }
  return hipErrorInvalidValue;
}

template <typename T, PairEpilogue EPI>
hipError_t run_pair(const PairArgs& g, bool symmetric, hipStream_t s) {
  const PairCut c = cut_pair(g.rows, g.cols, g.steps, symmetric);
  if (c.side == 64) return run_tiles<T, 1, 4, EPI>(g, c, s);
  return run_tiles<T, 2, 1, EPI>(g, c, s);
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
  auto blocks = [&](size_t at, int64_t across) { return Blocks{reinterpret_cast<f16*>(base + at), across}; };
  const int64_t n_blocks = p.n_pad / 32, m_blocks = p.m_pad / 32;
  const Blocks x[2] = {blocks(p.x[0], m_blocks), blocks(p.x[1], m_blocks)};
  const Blocks xt[2] = {blocks(p.xt[0], n_blocks), blocks(p.xt[1], n_blocks)};
  const Blocks gram = blocks(p.a, n_blocks), poly = blocks(p.p, n_blocks);

  Source<T> u{static_cast<const T*>(a.x), a.x_ld, a.m, a.m_ld, a.momentum, a.nesterov};
  squares_kernel<T><<<uint32_t(kSumBlocks), kThreads, 0, s>>>(u, a.m, a.rows, a.cols, sums);
  hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;
  const dim3 grid(uint32_t(p.m_pad / 64), uint32_t(p.n_pad / 64));
  prepare_kernel<T><<<grid, kThreads, 0, s>>>(u, p.n, p.m, p.tall, sums, it, factors, x[0], xt[0]);
  if ((e = hipGetLastError()) != hipSuccess) return e;

  for (int k = 0; k < a.steps; ++k) {
    const int now = k % 2, next = 1 - now;
    PairArgs g{};
    g.partial = reinterpret_cast<float*>(base + p.partial);
    g.a = g.b = x[now];  // A = X X^T
    g.rows = g.cols = p.n_pad;
    g.steps = m_blocks;
    g.factors = &factors[k].gram;
    g.out = gram;
    if ((e = run_pair<T, PAIR_BLOCKS>(g, true, s)) != hipSuccess) return e;
    g.a = g.b = g.d = gram;  // P = b A + c A A^T
    g.steps = n_blocks;
    g.factors = &factors[k].square;
    g.out = poly;
    if ((e = run_pair<T, PAIR_BLOCKS>(g, true, s)) != hipSuccess) return e;
    g.factors = &factors[k].apply;  // a X + P X
    if (k + 1 < a.steps) {
      g.a = poly;
      g.b = xt[now];
      g.d = x[now];
      g.cols = p.m_pad;
      g.out = x[next];
      g.across = xt[next];
      if ((e = run_pair<T, PAIR_BLOCKS>(g, false, s)) != hipSuccess) return e;
      continue;
    }
    // the result, or its transpose: rows of a tall one are columns of X
    g.a = p.tall ? xt[now] : poly;
    g.b = p.tall ? poly : xt[now];
    g.d = p.tall ? xt[now] : x[now];
    (p.tall ? g.rows : g.cols) = p.m_pad;
    g.y = a.y;
    g.y_ld = a.y_ld;
    g.y_rows = a.rows;
    g.y_cols = a.cols;
    g.decay = a.decay;
    g.step = a.step;
    e = a.m ? run_pair<T, PAIR_STEP>(g, false, s) : run_pair<T, PAIR_OUT>(g, false, s);
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
