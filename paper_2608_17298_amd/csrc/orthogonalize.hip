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
// result is float32's (2-norm 2.4e-6 off at 256 x 256, as the same steps in float32
// are).  With operands rounded once to float16 it is 1e-3 to 4e-3 off, more than
// bfloat16's rounding of the result.  A large product runs at 153 TFLOP/s in float32 on
// this card and at 1106 in float16, so three of those take less than half the time.
// a X is added in float: inside P it would double the error.
#include "orthogonalize_small.h"
#include "tile.h"

namespace gart {
namespace {

constexpr int kThreads = 256;

// The `count` elements from (r, c) of what is orthogonalised as floats, 0 behind
// them.  STEP: m is stepped there first, m <- momentum m + g.
template <typename T, bool MOMENTUM, bool STEP>
__device__ __forceinline__ void load_source(float (&w)[Pack<T>::N], const Source<T>& u, float* m, int64_t r, int64_t c,
                                            int count) {
  constexpr int V = Pack<T>::N;
  const Pack<T> x = load_some(u.x + r * u.ld + c, count);
#pragma unroll
  for (int e = 0; e < V; ++e) w[e] = float(x.v[e]);
  if constexpr (MOMENTUM) {
    float* at = m + r * u.m_ld + c;
#pragma unroll
    for (int h = 0; h < V / 4; ++h) {
      if (count <= 4 * h) continue;
      Pack<float> f = load_some(at + 4 * h, count - 4 * h);
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const float g = w[4 * h + e];
        if (STEP) f.v[e] = fmaf(u.momentum, f.v[e], g);
        w[4 * h + e] = u.nesterov ? fmaf(u.momentum, f.v[e], g) : f.v[e];
      }
      if (STEP) store_some(at + 4 * h, f, count - 4 * h);
    }
  }
}

// Steps m, if there is one, and sums the squares of what is to be orthogonalised in
// 64 bits: float's squares would overflow from 2e19 on.  A row is 2^log_lanes
// threads', a pack each at a time.
template <typename T, bool MOMENTUM>
__global__ __launch_bounds__(kThreads) void squares_kernel(const Source<T> u, float* __restrict__ m, int64_t rows,
                                                           int64_t cols, int log_lanes, double* __restrict__ sums) {
  constexpr int V = Pack<T>::N;
  __shared__ double s[kThreads / 64];
  const int lanes = 1 << log_lanes, lane = threadIdx.x % lanes, high = kThreads >> log_lanes;
  double t = 0.0;
  for (int64_t r = int64_t(blockIdx.x) * high + (threadIdx.x >> log_lanes); r < rows; r += int64_t(gridDim.x) * high)
    for (int64_t c = int64_t(lane) * V; c < cols; c += int64_t(lanes) * V) {
      float w[V];
      load_source<T, MOMENTUM, true>(w, u, m, r, c, int(min(int64_t(V), cols - c)));
#pragma unroll
      for (int e = 0; e < V; ++e) t = fma(double(w[e]), double(w[e]), t);
    }
#pragma unroll
  for (int off = 32; off > 0; off >>= 1) t += __shfl_xor(t, off);
  if (threadIdx.x % 64 == 0) s[threadIdx.x / 64] = t;
  __syncthreads();
  if (threadIdx.x == 0) sums[blockIdx.x] = (s[0] + s[1]) + (s[2] + s[3]);
}

// Of a tile in LDS, element (i, j) at tile[i * pitch + j], into blocks: those of rows
// i, or, transposed, of rows j.  Values are split into two parts.
constexpr int kTilePitch = 64 + 4;
template <int SIDE, bool TRANSPOSED>
__device__ __forceinline__ void store_blocks(const float* tile, const Blocks& to, int64_t row0, int64_t col0, int lane,
                                             int first, int step) {
  const int r = lane % 16, g = lane / 16;
  constexpr int DEEP = SIDE / 32;
  for (int b = first; b < SIDE / 16 * DEEP; b += step) {
    const int row = 16 * (b / DEEP) + r, k = 32 * (b % DEEP) + 8 * g;
    Pack<f16> high, low;
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      f16 h, l;
      split(TRANSPOSED ? tile[(k + e) * kTilePitch + row] : tile[row * kTilePitch + k + e], h, l);
      high.v[e] = h;
      low.v[e] = l;
    }
    f16* block = to.at(row0 / 16 + b / DEEP, col0 / 32 + b % DEEP) + lane * 8;
    store_pack(block, high);
    store_pack(block + Blocks::kBlock, low);
  }
}

// X and its transpose, zero in the padding, from u over its norm: 64 x 64 elements a
// block; and the steps' factors, by the first one.  Bound by bytes and the two orders
// of the stores: 1024 x 4096 bf16 in 15 us.
template <typename T, bool MOMENTUM>
__global__ __launch_bounds__(kThreads) void prepare_kernel(const Source<T> u, int64_t rows, int64_t cols, bool tall,
                                                           const double* __restrict__ sums, int count,
                                                           const Iteration it, StepFactors* __restrict__ factors,
                                                           const Blocks x, const Blocks xt) {
  constexpr int V = Pack<T>::N, ACROSS = 64 / V, EACH = 64 * ACROSS / kThreads;  // packs a row, and a thread
  __shared__ double s_sum[kThreads / 64];
  __shared__ __attribute__((aligned(16))) float s_tile[64 * kTilePitch];
  const int lane = threadIdx.x % 64, wave = threadIdx.x / 64;
  const int64_t tiles = (cols + 63) / 64, r0 = blockIdx.x / tiles * 64, c0 = blockIdx.x % tiles * 64;
  float w[EACH][V];  // all asked for first
#pragma unroll
  for (int q = 0; q < EACH; ++q) {
    const int at = q * kThreads + threadIdx.x;
    const int64_t r = r0 + at / ACROSS, c = c0 + at % ACROSS * V;
    const int here = r < rows ? int(max(int64_t(0), min(int64_t(V), cols - c))) : 0;
    load_source<T, MOMENTUM, false>(w[q], u, const_cast<float*>(u.m), r, c, here);
  }
  double t = 0.0;
  for (int q = threadIdx.x; q < count; q += kThreads) t += sums[q];
#pragma unroll
  for (int off = 32; off > 0; off >>= 1) t += __shfl_xor(t, off);
  if (lane == 0) s_sum[wave] = t;
  __syncthreads();
  const double size = sqrt((s_sum[0] + s_sum[1]) + (s_sum[2] + s_sum[3]));
  bool tiny;
  const double inv = first_scale(it, size, tiny);
  if (blockIdx.x == 0) {
    if (!tiny) {
      if (threadIdx.x < it.steps) factors[threadIdx.x] = it.of_one.step[threadIdx.x];
    } else if (threadIdx.x == 0) {
      float first;
      step_factors(it.a, it.b, it.c, it.steps, size / (size + double(it.eps)), &first, factors);
    }
  }
#pragma unroll
  for (int q = 0; q < EACH; ++q) {
    const int at = q * kThreads + threadIdx.x, r = at / ACROSS, c = at % ACROSS * V;
    const int64_t left = r0 + r < rows ? cols - c0 - c : 0;  // the padding stays 0 whatever the norm
#pragma unroll
    for (int h = 0; h < V / 4; ++h) {
      f32x4 f;
#pragma unroll
      for (int e = 0; e < 4; ++e) f[e] = 4 * h + e < left ? float(double(w[q][4 * h + e]) * inv) : 0.0f;
      *reinterpret_cast<f32x4*>(s_tile + r * kTilePitch + c + 4 * h) = f;
    }
  }
  __syncthreads();
  // the rows of x are those of X, or of its transpose
  store_blocks<64, false>(s_tile, tall ? xt : x, r0, c0, lane, wave, kThreads / 64);
  store_blocks<64, true>(s_tile, tall ? x : xt, c0, r0, lane, wave, kThreads / 64);
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
  TileOrder order;      // symmetric: C is, tiles above the diagonal are stored on both sides of it
  int tiles;            // launched for them, for each part of k
  int parts;
  float* partial;       // their sums
  const float* factors; // alpha, beta
  Blocks out, across;   // PAIR_BLOCKS: C and, unless it is symmetric, its transpose
  void* y;              // else: the result
  int64_t y_ld, y_rows, y_cols;
  float decay, step;    // PAIR_STEP: y -= decay y + step C
};

// The sums of a product, two ways:
//
//  - Waves that split k (WK of them).  Each has all FRAG x FRAG fragments of the tile
//    and takes every WK-th block of k straight from memory: nothing is shared, so
//    nothing passes through LDS.  Two sets of fragments are on their way while one is
//    multiplied; the waves meet when their sums are joined.  Bound by the bytes a CU
//    takes in (100 a ns from its cache, 65 from another die's), for products with few
//    tiles.
//  - Two groups of W x W waves of 64 x 64 that share the operands in LDS (tiles of
//    128) and take every other block of k: two waves a SIMD, of which one multiplies
//    while the other reads its fragments (one wave that reads ahead instead: 1024 x
//    1024 -> 4096 39 us, these 34 on the same card).
template <int FRAG>
struct Fragments {
  Pack<f16>::V ah[FRAG], al[FRAG], bh[FRAG], bl[FRAG];
};
template <int FRAG>
__device__ __forceinline__ void multiply(f32x4 (&sum)[FRAG][FRAG], const Fragments<FRAG>& f) {
#pragma unroll
  for (int p = 0; p < 3; ++p)
#pragma unroll
    for (int i = 0; i < FRAG; ++i)
#pragma unroll
      for (int j = 0; j < FRAG; ++j)
        sum[i][j] = Mfma<f16>::run(p == 0 ? f.bl[j] : f.bh[j], p == 1 ? f.al[i] : f.ah[i], sum[i][j]);
}

template <int FRAG, int WK, typename F>
__device__ __forceinline__ void split_sums(f32x4 (&sum)[FRAG][FRAG], const PairArgs& g, int64_t i0, int64_t j0, int k0,
                                           int k1, int lane, F&& meanwhile) {
  const int64_t a_row = g.a.across * Blocks::kPair, b_row = g.b.across * Blocks::kPair;
  const f16* a = g.a.at(i0 / 16, k0) + lane * 8;
  const f16* b = g.b.at(j0 / 16, k0) + lane * 8;
  Fragments<FRAG> set[3];
  auto load = [&](Fragments<FRAG>& f, int n) {  // past the end the last one again
    const int64_t at = int64_t(min(n, (k1 - 1 - k0) / WK)) * (WK * Blocks::kPair);
#pragma unroll
    for (int i = 0; i < FRAG; ++i) {
      f.ah[i] = *reinterpret_cast<const Pack<f16>::V*>(a + i * a_row + at);
      f.al[i] = *reinterpret_cast<const Pack<f16>::V*>(a + i * a_row + at + Blocks::kBlock);
      f.bh[i] = *reinterpret_cast<const Pack<f16>::V*>(b + i * b_row + at);
      f.bl[i] = *reinterpret_cast<const Pack<f16>::V*>(b + i * b_row + at + Blocks::kBlock);
    }
    __builtin_amdgcn_sched_barrier(0);  // asked for here, not where they are used
  };
  auto product = [&](const Fragments<FRAG>& f) {
    multiply<FRAG>(sum, f);
    __builtin_amdgcn_sched_barrier(0);
  };
  const int count = (k1 - k0 + WK - 1) / WK;
  load(set[0], 0);
  load(set[1], 1);
  meanwhile();
  int n = 0;
  for (; n + 2 < count; n += 3) {
    load(set[2], n + 2);
    product(set[0]);
    load(set[0], n + 3);
    product(set[1]);
    load(set[1], n + 4);
    product(set[2]);
  }
  if (n < count) product(set[0]);
  if (n + 1 < count) product(set[1]);
}

// Wave `wave` of group `group`: every kGroups-th block of k.
constexpr int kGroups = 2, kStages = 2;
template <int W>
__device__ __forceinline__ void shared_sums(f32x4 (&sum)[4][4], const PairArgs& g, int64_t ti, int64_t tj, int k0, int k1,
                                            int group, int wave, int lane, f16* lds) {
  // a stage: kGroups blocks of k, each 4 W row tiles of A, then of B, pairs of blocks
  constexpr int TILES = 4 * W, BLOCK = 2 * TILES * Blocks::kPair, STAGE = kGroups * BLOCK, MINE = TILES / (W * W);
  static_assert(TILES % (W * W) == 0, "whole tiles a wave");
  typedef const __attribute__((address_space(1))) uint32_t* global_ptr;
  typedef __attribute__((address_space(3))) uint32_t* lds_ptr;
  const int64_t a_last = g.rows / 16 - 1, b_last = g.cols / 16 - 1;  // tiles past the end: the last one again
  const f16 *a[MINE], *b[MINE];
#pragma unroll
  for (int u = 0; u < MINE; ++u) {
    a[u] = g.a.at(min(ti * TILES + wave * MINE + u, a_last), 0) + lane * 8;
    b[u] = g.b.at(min(tj * TILES + wave * MINE + u, b_last), 0) + lane * 8;
  }
  f16* mine = lds + group * BLOCK;
  auto fetch = [&](int h, int k) {  // past the end the last one again: it is not used
    f16* to = mine + h * STAGE + wave * MINE * Blocks::kPair;
    const int64_t at = int64_t(min(k, k1 - 1)) * Blocks::kPair;
#pragma unroll
    for (int u = 0; u < MINE; ++u)
#pragma unroll
      for (int half = 0; half < 2; ++half) {
        const int64_t off = half * Blocks::kBlock;
        __builtin_amdgcn_global_load_lds((global_ptr)(a[u] + at + off), (lds_ptr)(to + u * Blocks::kPair + off), 16, 0, 0);
        __builtin_amdgcn_global_load_lds((global_ptr)(b[u] + at + off),
                                         (lds_ptr)(to + (TILES + u) * Blocks::kPair + off), 16, 0, 0);
      }
  };
  const int wi = wave / W, wj = wave % W;
  int h = 0;
  fetch(0, k0 + group);
  for (int k = k0; k < k1; k += kGroups, h ^= 1) {
    // this wave's part of the stage has landed, and it has read the one before
    asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)" ::: "memory");
    __builtin_amdgcn_s_barrier();  // so has everyone's, and have they
    asm volatile("" ::: "memory");
    if (k + kGroups < k1) fetch(h ^ 1, k + kGroups + group);
    if (k + group < k1) {
      const f16* from = mine + h * STAGE + lane * 8;
      Fragments<4> f;
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const f16* p = from + (wi * 4 + i) * Blocks::kPair;
        const f16* q = from + (TILES + wj * 4 + i) * Blocks::kPair;
        f.ah[i] = *reinterpret_cast<const Pack<f16>::V*>(p);
        f.al[i] = *reinterpret_cast<const Pack<f16>::V*>(p + Blocks::kBlock);
        f.bh[i] = *reinterpret_cast<const Pack<f16>::V*>(q);
        f.bl[i] = *reinterpret_cast<const Pack<f16>::V*>(q + Blocks::kBlock);
      }
      multiply<4>(sum, f);
    }
  }
}

// A tile of 16 FRAG W on a side.  JOIN: the sums of k are those of g.parts parts.
// 1024 x 4096: X X^T in seven parts 20 us and their join 9, A A 12, P X 35, of which 10
// are its stores and 31 % matrix instructions; its LDS reads take as long as those.
template <typename T, int FRAG, int W, int WK, PairEpilogue EPI, bool JOIN>
__global__ __launch_bounds__(64 * (JOIN ? 1 : W * W) * WK, 1) void pair_kernel(const PairArgs g) {
  constexpr int PLACES = JOIN ? 1 : W * W;  // tiles of waves in a block: a join has one, to have more blocks
  constexpr int THREADS = 64 * W * W * WK, SIDE = 16 * FRAG;
  constexpr bool SPLIT = W == 1;
  static_assert(SPLIT ? WK == 4 : FRAG == 4 && WK == kGroups, "four waves of one tile, or two groups of tiles of 64");
  // 16 x 16 tiles of a wave's result: its share of FRAG by FRAG
  constexpr int RJ = FRAG * FRAG / WK < FRAG ? FRAG * FRAG / WK : FRAG, RI = FRAG * FRAG / WK / RJ;
  constexpr int SUMS = JOIN ? 0 : SPLIT ? WK * SIDE * SIDE : kStages * kGroups * 2 * 4 * W * Blocks::kPair / 2;  // floats
  constexpr int TILE = EPI == PAIR_BLOCKS ? PLACES * SIDE * kTilePitch : 4;
  __shared__ __attribute__((aligned(16))) float lds[SUMS > TILE ? SUMS : TILE];
  const int lane = threadIdx.x % 64, wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64);
  const int at_xcd = int(xcd_tile(blockIdx.x, gridDim.x)), which = JOIN ? at_xcd / (W * W) : at_xcd;
  const int part = which / g.tiles;  // 0 but for PAIR_PART
  int ti, tj;
  if (!find_tile(g.order, which - part * g.tiles, ti, tj)) return;
  const int wk = wave / PLACES, place = JOIN ? at_xcd % (W * W) : wave % PLACES, wi = place / W, wj = place % W;
  const int tid = (wk * W * W + place) * 64 + lane;  // of the block that sums
  const int64_t i0 = (int64_t(ti) * W + wi) * SIDE, j0 = (int64_t(tj) * W + wj) * SIDE;
  const bool inside = is_result(g.order, g.rows, g.cols, i0, j0);
  const int first_i = wk * RI * RJ / FRAG, first_j = wk * RI * RJ % FRAG;
  const int r = lane % 16, g4 = lane / 16;
  typedef f16 f16x4 __attribute__((ext_vector_type(4)));
  // A lane has four consecutive columns of a row; of D they are half a piece.
  auto d_at = [&](int i, int j) {
    const int row = 16 * (first_i + i), col = 16 * (first_j + j) + 4 * g4;
    return g.d.at((i0 + row) / 16, (j0 + col) / 32) + (((j0 + col) % 32) / 8 * 16 + r) * 8 + col % 8;
  };
  f16x4 dh[RI][RJ], dl[RI][RJ];
  float alpha, beta;
  // What the result takes besides the sums, asked for before they are formed.
  auto others = [&]() {
    if constexpr (EPI != PAIR_PART) {
      alpha = g.factors[0];
      beta = g.factors[1];
      if (g.d.data && inside) {
#pragma unroll
        for (int i = 0; i < RI; ++i)
#pragma unroll
          for (int j = 0; j < RJ; ++j) {
            dh[i][j] = *reinterpret_cast<const f16x4*>(d_at(i, j));
            dl[i][j] = *reinterpret_cast<const f16x4*>(d_at(i, j) + Blocks::kBlock);
          }
      }
    }
  };

  f32x4 acc[RI][RJ];
  if constexpr (JOIN) {
    others();
#pragma unroll
    for (int i = 0; i < RI; ++i)
#pragma unroll
      for (int j = 0; j < RJ; ++j) acc[i][j] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
    // Four parts' sums are asked for before the first is added; past the end the last one again.
    constexpr int AHEAD = 4;
    f32x4 next[AHEAD][RI][RJ];
    auto load = [&](f32x4(&to)[RI][RJ], int q) {
      const float* from = g.partial + (int64_t(min(q, g.parts - 1)) * g.tiles + which) * (THREADS * RI * RJ * 4) + tid * 4;
#pragma unroll
      for (int i = 0; i < RI; ++i)
#pragma unroll
        for (int j = 0; j < RJ; ++j) to[i][j] = *reinterpret_cast<const f32x4*>(from + (i * RJ + j) * THREADS * 4);
    };
    for (int q = 0; q < g.parts; q += AHEAD) {
#pragma unroll
      for (int h = 0; h < AHEAD; ++h) load(next[h], q + h);
      __builtin_amdgcn_sched_barrier(0);
#pragma unroll
      for (int h = 0; h < AHEAD; ++h) {
        if (q + h >= g.parts) break;
#pragma unroll
        for (int i = 0; i < RI; ++i)
#pragma unroll
          for (int j = 0; j < RJ; ++j) acc[i][j] += next[h][i][j];
      }
    }
  } else {
    f32x4 sum[FRAG][FRAG];
#pragma unroll
    for (int i = 0; i < FRAG; ++i)
#pragma unroll
      for (int j = 0; j < FRAG; ++j) sum[i][j] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
    const int parts = EPI == PAIR_PART ? g.parts : 1;
    const int k0 = int(g.steps * part / parts), k1 = int(g.steps * (part + 1) / parts);
    if constexpr (!SPLIT) {
      shared_sums<W>(sum, g, ti, tj, k0, k1, wk, place, lane, reinterpret_cast<f16*>(lds));
      others();
      __syncthreads();
    } else if (k0 + wk < k1) {
      split_sums<FRAG, WK>(sum, g, i0, j0, k0 + wk, k1, lane, others);
    } else {
      others();
    }
    // each of the WK waves takes its share of the others' tiles
    constexpr int SHARE = RI * RJ, ALL = FRAG * FRAG;
    float* at = lds + place * (WK * ALL * 256) + lane * 4;
#pragma unroll
    for (int q = 0; q < ALL; ++q)
      if (q / SHARE != wk) *reinterpret_cast<f32x4*>(at + (wk * ALL + q) * 256) = sum[q / FRAG][q % FRAG];
    __syncthreads();
#pragma unroll
    for (int q = 0; q < SHARE; ++q) {
      f32x4 t = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
      for (int w = 0; w < WK; ++w) {
        f32x4 own = t;
#pragma unroll
        for (int v = 0; v < WK; ++v)
          if (v == w) own = sum[(v * SHARE + q) / FRAG][(v * SHARE + q) % FRAG];
        t += w == wk ? own : *reinterpret_cast<const f32x4*>(at + (w * ALL + wk * SHARE + q) * 256);
      }
      arrive(t);  // the compiler moved these reads behind the barrier, where the tile is written over them
      acc[q / RJ][q % RJ] = t;
    }
    __syncthreads();
  }

  if constexpr (EPI == PAIR_PART) {
    float* to = g.partial + int64_t(which) * (THREADS * RI * RJ * 4) + tid * 4;
#pragma unroll
    for (int i = 0; i < RI; ++i)
#pragma unroll
      for (int j = 0; j < RJ; ++j) *reinterpret_cast<f32x4*>(to + (i * RJ + j) * THREADS * 4) = acc[i][j];
    return;
  }

  float* tile = lds + (JOIN ? 0 : place) * SIDE * kTilePitch;
  if (inside) {
#pragma unroll
    for (int i = 0; i < RI; ++i) {
      const int row = 16 * (first_i + i) + r;
#pragma unroll
      for (int j = 0; j < RJ; ++j) {
        const int col = 16 * (first_j + j) + 4 * g4;
        f32x4 c = alpha * acc[i][j];
        if (g.d.data) {
#pragma unroll
          for (int e = 0; e < 4; ++e) c[e] = fmaf(beta, float(dh[i][j][e]) + float(dl[i][j][e]), c[e]);
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
    store_blocks<SIDE, false>(tile, g.out, i0, j0, lane, wk, WK);
    if (!g.order.symmetric)
      store_blocks<SIDE, true>(tile, g.across, j0, i0, lane, WK - 1 - wk, WK);
    else if (i0 != j0)
      store_blocks<SIDE, true>(tile, g.out, j0, i0, lane, WK - 1 - wk, WK);
  }
}

template <typename T, int FRAG, int W, int WK, PairEpilogue EPI>
hipError_t run_tiles(PairArgs g, const PairCut& c, hipStream_t s) {
  g.order = tile_order(g.rows, g.cols, c.side, c.symmetric);
  g.parts = c.parts;
  g.tiles = int(blocks_of(g.rows, g.cols, c.side, c.symmetric));
  constexpr int THREADS = 64 * W * W * WK;
  if (c.parts == 1) {
    pair_kernel<T, FRAG, W, WK, EPI, false><<<uint32_t(g.tiles), THREADS, 0, s>>>(g);
    return hipGetLastError();
  }
  if constexpr (EPI == PAIR_BLOCKS) {
    pair_kernel<T, FRAG, W, WK, PAIR_PART, false><<<uint32_t(g.tiles * c.parts), THREADS, 0, s>>>(g);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
    pair_kernel<T, FRAG, W, WK, PAIR_BLOCKS, true><<<uint32_t(g.tiles * W * W), 64 * WK, 0, s>>>(g);
    return hipGetLastError();
  }
  return hipErrorInvalidValue;
}

template <typename T, PairEpilogue EPI>
hipError_t run_pair(const PairArgs& g, bool symmetric, hipStream_t s) {
  const PairCut c = cut_pair(g.rows, g.cols, g.steps, symmetric);
  if (c.side == 32) return run_tiles<T, 2, 1, 4, EPI>(g, c, s);
  if (c.side == 64) return run_tiles<T, 4, 1, 4, EPI>(g, c, s);
  return run_tiles<T, 4, 2, kGroups, EPI>(g, c, s);
}

template <typename T>
hipError_t run(const OrthogonalizeArgs& a, hipStream_t s) {
  if (a.rows <= 0 || a.cols <= 0) return hipSuccess;
  const MatrixPlan p = matrix_plan(a.rows, a.cols);
  Iteration it{a.a, a.b, a.c, a.eps, a.steps, {}};
  if (!step_factors(a.a, a.b, a.c, a.steps, 1.0, &it.of_one.x, it.of_one.step)) return hipErrorInvalidValue;
  if (small_fits(p)) return run_small<T>(a, p, it, s);
  char* base = static_cast<char*>(a.scratch);
  double* sums = reinterpret_cast<double*>(base + p.sums);
  StepFactors* factors = reinterpret_cast<StepFactors*>(base + p.factors);
  auto blocks = [&](size_t at, int64_t across) { return Blocks{reinterpret_cast<f16*>(base + at), across}; };
  const int64_t n_blocks = p.n_pad / 32, m_blocks = p.m_pad / 32;
  const Blocks x[2] = {blocks(p.x[0], m_blocks), blocks(p.x[1], m_blocks)};
  const Blocks xt[2] = {blocks(p.xt[0], n_blocks), blocks(p.xt[1], n_blocks)};
  const Blocks gram = blocks(p.a, n_blocks), poly = blocks(p.p, n_blocks);

  Source<T> u{static_cast<const T*>(a.x), a.x_ld, a.m, a.m_ld, a.momentum, a.nesterov};
  int log_lanes = 0;
  while (log_lanes < 8 && int64_t(Pack<T>::N) << log_lanes < a.cols) ++log_lanes;
  const int count = int(std::min<int64_t>(kSumBlocks, ceil_div64(a.rows << log_lanes, kThreads)));
  if (a.m)
    squares_kernel<T, true><<<uint32_t(count), kThreads, 0, s>>>(u, a.m, a.rows, a.cols, log_lanes, sums);
  else
    squares_kernel<T, false><<<uint32_t(count), kThreads, 0, s>>>(u, nullptr, a.rows, a.cols, log_lanes, sums);
  hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;
  const uint32_t grid = uint32_t(p.n_pad / 64 * (p.m_pad / 64));
  if (a.m)
    prepare_kernel<T, true><<<grid, kThreads, 0, s>>>(u, a.rows, a.cols, p.tall, sums, count, it, factors, x[0], xt[0]);
  else
    prepare_kernel<T, false><<<grid, kThreads, 0, s>>>(u, a.rows, a.cols, p.tall, sums, count, it, factors, x[0], xt[0]);
  if ((e = hipGetLastError()) != hipSuccess) return e;

  for (int k = 0; k < a.steps; ++k) {
    const int now = k % 2, next = 1 - now;
    PairArgs g{};
    g.partial = reinterpret_cast<float*>(base + p.x[next]);
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
