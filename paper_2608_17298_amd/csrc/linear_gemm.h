// Tiled products of the linear layer and its gradient, for one element type.
//
// C[i,j] = sum_k A(i,k) B(j,k) on 16x16 matrix-core tiles, sums in float.  B's
// tile is the matrix instruction's first operand, so a lane holds consecutive
// j of one i and stores along rows.  An operand is either k-contiguous (x and
// W of the forward) or i-contiguous (the gradient's, whose sums run over rows
// or outputs): the first kind lies in LDS as rows of 128 bytes, the second as
// lines across k, and its 16-bit fragments are read with the transposing LDS
// load.  16-byte (rows) or 32-byte (lines) pieces trade places by row or line,
// so that lanes that read together meet different banks.
//
// Large products are bound by the matrix cores: 4096 x 1024 -> 4096 f16 with
// gelu and residual takes 43 us (800 TFLOP/s), of which about 12 are the first
// loads and the outputs; each further 1024 of k costs 26 us (1300 TFLOP/s).
// Products with short sums or few tiles are bound by the way from memory, so
// two steps of k are on the way while one is multiplied.
#pragma once

#include <algorithm>

#include "linear.h"
#include "linear_small.h"
#include "tile.h"

namespace gart {
namespace {

// What is done with the products.
enum Epilogue {
  EPI_FORWARD,  // y = act(c + bias) + residual
  EPI_DZ,       // dz = dl act'(c + bias), and its column sums per tile of rows
  EPI_STORE,    // y = c
  EPI_PARTIAL   // float c of one part of the sum
};

struct GemmArgs {
  const void *a, *b;
  int64_t a_ld, b_ld;
  int64_t a_low;  // A is dz: elements from its high parts to the low ones, or 0
  int64_t rows, cols, depth;  // of C, and the length of the sums
  int64_t part;               // length of one part of the sums (EPI_PARTIAL: blockIdx.z)
  int64_t tiles_i, tiles_j;
  gart_activation act;
  const void *bias, *extra;  // extra: residual or dl
  int64_t extra_ld;
  void* out;
  int64_t out_ld, out_low;  // out_low: EPI_DZ, as a_low
  float* sums;  // EPI_DZ: [tiles_i, cols] column sums, or NULL
};

// TI x TJ tiles a wave, WI x WJ waves a block.  DIRECT: both operands go
// straight from memory into LDS, which needs 16-byte aligned rows and whole
// steps of k; otherwise they pass through registers.  PARTS: A is dz in two
// parts (split_dz), the low ones g.a_low elements behind the high ones.
template <typename T, bool AKC, bool BKC, int TI, int TJ, int WI, int WJ, bool DIRECT, Epilogue EPI, bool PARTS>
__global__ __launch_bounds__(64 * WI * WJ, PARTS ? 2 : 1) void gemm_kernel(const GemmArgs g) {
  constexpr int THREADS = 64 * WI * WJ;
  using TA = Tile<T, AKC, 16 * TI * WI, WI * WJ, false>;
  using TB = Tile<T, BKC, 16 * TJ * WJ, WI * WJ, true>;
  constexpr int BI = 16 * TI * WI, BJ = 16 * TJ * WJ, V = Pack<T>::N;
  // Both parts of a step meet B's fragments at a time, in one LDS buffer, so that two blocks still fit a CU (one part
  // after the other, in two buffers: gradient of 60000 x 300 -> 400 bf16 381 us, so 294).  With the second launch bound
  // the sums stay out of the accumulation registers, which no fma reaches (f16: 405 us, so 304).
  constexpr bool BOTH = PARTS && !DIRECT;
  constexpr int A_LOW = TA::ELEMS + TB::ELEMS, ELEMS = A_LOW + (BOTH ? TA::ELEMS : 0);
  __shared__ __attribute__((aligned(16))) T lds[BOTH ? 1 : 2][ELEMS];
  __shared__ float s_sum[EPI == EPI_DZ ? WI : 1][EPI == EPI_DZ ? BJ : 1];

  const int tid = threadIdx.x, lane = tid % 64, wave = __builtin_amdgcn_readfirstlane(tid / 64);
  const int wi = wave / WJ, wj = wave % WJ;
  const int64_t tile = xcd_tile(blockIdx.x, g.tiles_i * g.tiles_j);
  const int64_t i0 = tile / g.tiles_j * BI, j0 = tile % g.tiles_j * BJ;
  const int64_t k0 = EPI == EPI_PARTIAL ? int64_t(blockIdx.z) * g.part : 0;
  const int64_t k1 = EPI == EPI_PARTIAL ? min(g.depth, k0 + g.part) : g.depth;
  const T* pa = static_cast<const T*>(g.a);
  const T* pb = static_cast<const T*>(g.b);

  f32x4 acc[TI][TJ];
#pragma unroll
  for (int i = 0; i < TI; ++i)
#pragma unroll
    for (int j = 0; j < TJ; ++j) acc[i][j] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};

  auto multiply = [&](const T* la, const T* lb) {
#pragma unroll
    for (int s = 0; s < 2; ++s) {
      typename Pack<T>::V fa[TI], fa_low[TI], fb[TJ];
#pragma unroll
      for (int j = 0; j < TJ; ++j) fb[j] = TB::fragment(lb, wj * TJ + j, s, lane);
#pragma unroll
      for (int i = 0; i < TI; ++i) {
        fa[i] = TA::fragment(la, wi * TI + i, s, lane);
        if (BOTH) fa_low[i] = TA::fragment(la + A_LOW, wi * TI + i, s, lane);
      }
#pragma unroll
      for (int i = 0; i < TI; ++i)
#pragma unroll
        for (int j = 0; j < TJ; ++j)
          acc[i][j] = BOTH ? mfma_dz<T>(fb[j], fa[i], fa_low[i], acc[i][j]) : Mfma<T>::run(fb[j], fa[i], acc[i][j]);
    }
  };
  const int64_t a_step = TA::stride(g.a_ld), b_step = TB::stride(g.b_ld), whole = (k1 - k0) / kStep<T>;
  TA ta;
  TB tb;
  if constexpr (DIRECT) {
    ta.template aim<true>(pa, g.a_ld, i0, g.rows, k0, tid);
    tb.template aim<true>(pb, g.b_ld, j0, g.cols, k0, tid);
    // PARTS: the sums run over dz's low parts first, whose scale is then taken back, and then over the high ones
    const int64_t steps = PARTS ? 2 * whole : whole;
    auto fetch = [&](int h, int64_t n) {
      const int64_t at = PARTS && n >= whole ? n - whole : n;
      ta.fetch(lds[h], at * a_step + (PARTS && n < whole ? g.a_low : 0), wave);
      tb.fetch(lds[h] + TA::ELEMS, at * b_step, wave);
    };
    if (steps > 0) fetch(0, 0);
    for (int64_t n = 0; n < steps; ++n) {
      asm volatile("s_waitcnt vmcnt(0)" ::: "memory");  // this wave's part of the buffer has landed
      __syncthreads();                                  // everyone's has, and the other buffer has been read
      if (n + 1 < steps) fetch((n + 1) & 1, n + 1);
      if constexpr (PARTS && kDzLow<T> != 1.0f) {
        if (n == whole) {
#pragma unroll
          for (int i = 0; i < TI; ++i)
#pragma unroll
            for (int j = 0; j < TJ; ++j) acc[i][j] *= 1.0f / kDzLow<T>;
        }
      }
      multiply(lds[n & 1], lds[n & 1] + TA::ELEMS);
    }
  } else if constexpr (PARTS) {
    const int64_t inner = TA::regular(i0, g.rows) && TB::regular(j0, g.cols) ? whole : 0;
    const int64_t steps = (k1 - k0 + kStep<T> - 1) / kStep<T>;
    if (inner > 0) {
      ta.template aim<false>(pa, g.a_ld, i0, g.rows, k0, tid);
      tb.template aim<false>(pb, g.b_ld, j0, g.cols, k0, tid);
    }
    Pack<T> ra[TA::PER_THREAD], ra_low[TA::PER_THREAD], rb[TB::PER_THREAD];
    auto load = [&](int64_t n) {
      if (n < inner) {
        ta.load(ra, n * a_step);
        ta.load(ra_low, n * a_step + g.a_low);
        tb.load(rb, n * b_step);
      } else if (n < steps) {
        const int64_t at = k0 + n * kStep<T>;
        TA::load_edge(ra, pa, g.a_ld, i0, g.rows, at, k1, tid);
        TA::load_edge(ra_low, pa + g.a_low, g.a_ld, i0, g.rows, at, k1, tid);
        TB::load_edge(rb, pb, g.b_ld, j0, g.cols, at, k1, tid);
      }
    };
    load(0);
    for (int64_t n = 0; n < steps; ++n) {
      TA::store(lds[0], ra, tid);
      TA::store(lds[0] + A_LOW, ra_low, tid);
      TB::store(lds[0] + TA::ELEMS, rb, tid);
      lds_barrier();
      load(n + 1);
      multiply(lds[0], lds[0] + TA::ELEMS);
      lds_barrier();  // the buffer has been read
    }
  } else {
    int64_t k = k0;
    if (whole > 0 && TA::regular(i0, g.rows) && TB::regular(j0, g.cols)) {
      // Two steps are on the way while one is multiplied: with few blocks a CU a
      // step is much shorter than the way from memory.
      ta.template aim<false>(pa, g.a_ld, i0, g.rows, k0, tid);
      tb.template aim<false>(pb, g.b_ld, j0, g.cols, k0, tid);
      Pack<T> ra[2][TA::PER_THREAD], rb[2][TB::PER_THREAD];
      auto load = [&](int h, int64_t n) {
        n = min(n, whole - 1);
        ta.load(ra[h], n * a_step);
        tb.load(rb[h], n * b_step);
      };
      auto step = [&](int h, int64_t n) {
        TA::store(lds[h], ra[h], tid);
        TB::store(lds[h] + TA::ELEMS, rb[h], tid);
        lds_barrier();  // also: the other buffer's readers are past it once all threads are here
        load(h, n + 2);
        multiply(lds[h], lds[h] + TA::ELEMS);
      };
      load(0, 0);
      load(1, 1);
      int64_t n = 0;
      for (; n + 1 < whole; n += 2) {
        step(0, n);
        step(1, n + 1);
      }
      if (n < whole) step(0, n);
      k += whole * kStep<T>;
      lds_barrier();
    }
    if (k < k1) {  // the last, partial step; or all of them
      Pack<T> ra[TA::PER_THREAD], rb[TB::PER_THREAD];
      auto load = [&](int64_t at) {
        TA::load_edge(ra, pa, g.a_ld, i0, g.rows, at, k1, tid);
        TB::load_edge(rb, pb, g.b_ld, j0, g.cols, at, k1, tid);
      };
      load(k);
      for (int h = 0; k < k1; k += kStep<T>, h ^= 1) {
        TA::store(lds[h], ra, tid);
        TB::store(lds[h] + TA::ELEMS, rb, tid);
        lds_barrier();
        if (k + kStep<T> < k1) load(k + kStep<T>);
        multiply(lds[h], lds[h] + TA::ELEMS);
      }
    }
  }

  // A lane's columns: V consecutive ones from each JQ tiles.
  constexpr int JQ = V / 4;
  const int r = lane % 16, q4 = lane / 16;
#pragma unroll
  for (int jq = 0; jq < TJ / JQ; ++jq) {
    const int jt = wj * TJ + jq * JQ;
    const int jl = JQ == 2 ? 32 * (jt / 2) + 8 * q4 : 16 * jt + 4 * q4;
    const int64_t j = j0 + jl;
    const int count = int(max(int64_t(0), min(int64_t(V), g.cols - j)));
    float b[V] = {};
    if constexpr (EPI == EPI_FORWARD || EPI == EPI_DZ) {
      if (g.bias && count > 0) {
        const Pack<T> p = load_some(static_cast<const T*>(g.bias) + j, count);
#pragma unroll
        for (int e = 0; e < V; ++e) b[e] = float(p.v[e]);
      }
    }
    float sum[V] = {};
#pragma unroll
    for (int i = 0; i < TI; ++i) {
      const int64_t row = i0 + 16 * (wi * TI + i) + r;
      if (row >= g.rows || count == 0) continue;
      float c[V];
#pragma unroll
      for (int e = 0; e < V; ++e) {
        c[e] = acc[i][jq * JQ + e / 4][e % 4];
        if (PARTS) c[e] *= 1.0f / kDzUnit<T>;
        c[e] += b[e];
      }
      if constexpr (EPI == EPI_PARTIAL) {
        float* out = static_cast<float*>(g.out) + (int64_t(blockIdx.z) * g.rows + row) * g.cols + j;
#pragma unroll
        for (int h = 0; h < V / 4; ++h) {
          Pack<float> f;
#pragma unroll
          for (int e = 0; e < 4; ++e) f.v[e] = c[4 * h + e];
          if (count > 4 * h) store_some(out + 4 * h, f, count - 4 * h);
        }
      } else {
        if constexpr (EPI == EPI_FORWARD) {
          with_activation(g.act, [&](auto act) {
#pragma unroll
            for (int e = 0; e < V; ++e) c[e] = activate<decltype(act)::value>(c[e]);
          });
        }
        if (EPI == EPI_DZ || (EPI == EPI_FORWARD && g.extra)) {
          const Pack<T> p = load_some(static_cast<const T*>(g.extra) + row * g.extra_ld + j, count);
          if constexpr (EPI == EPI_DZ) {
            with_activation(g.act, [&](auto act) {
#pragma unroll
              for (int e = 0; e < V; ++e) {
                c[e] = activate_grad<decltype(act)::value>(c[e], float(p.v[e]));
                if (e < count) sum[e] += c[e];
              }
            });
          } else {
#pragma unroll
            for (int e = 0; e < V; ++e) c[e] += float(p.v[e]);
          }
        }
        T* out = static_cast<T*>(g.out) + row * g.out_ld + j;
        auto put = [&](T* to, const Pack<T>& o) {
          if (DIRECT && count == V)
            store_past(to, o);  // large: it would push the operands out (4096 x 1024 -> 4096 f16: 50 us, past 44)
          else
            store_some(to, o, count);
        };
        Pack<T> o;
        if constexpr (EPI == EPI_DZ && sizeof(T) == 2) {
          if (g.out_low) {
            Pack<T> low;
            split_dz<T>(c, o, low);
            put(out, o);
            put(out + g.out_low, low);
            continue;
          }
        }
#pragma unroll
        for (int e = 0; e < V; ++e) o.v[e] = T(c[e]);
        put(out, o);
      }
    }
    if constexpr (EPI == EPI_DZ) {
#pragma unroll
      for (int e = 0; e < V; ++e) {
#pragma unroll
        for (int off = 1; off < 16; off <<= 1) sum[e] += __shfl_xor(sum[e], off);
        if (r == 0) s_sum[wi][jl + e] = sum[e];
      }
    }
  }
  if constexpr (EPI == EPI_DZ) {
    __syncthreads();
    if (g.sums)
      for (int j = tid; j < BJ && j0 + j < g.cols; j += THREADS) {
        float t = 0.0f;
#pragma unroll
        for (int w = 0; w < WI; ++w) t += s_sum[w][j];
        g.sums[tile / g.tiles_j * g.cols + j0 + j] = t;
      }
  }
}

// Column sums of m rows, one part of kSumRows rows a block: sums[part, n], or
// the result itself if there is one part.
template <typename T>
__global__ __launch_bounds__(256) void column_sums_kernel(const T* __restrict__ p, int64_t ld, int64_t m, int64_t n,
                                                          float* __restrict__ sums, T* __restrict__ out) {
  __shared__ float s[4][64];
  const int lane = threadIdx.x % 64, w = threadIdx.x / 64;
  const int64_t j = int64_t(blockIdx.y) * 64 + lane, r0 = int64_t(blockIdx.x) * kSumRows;
  float t = 0.0f;
  if (j < n)
    for (int64_t r = r0 + w; r < min(m, r0 + kSumRows); r += 4) t += float(p[r * ld + j]);
  s[w][lane] = t;
  __syncthreads();
  if (w > 0 || j >= n) return;
  t = (s[0][lane] + s[1][lane]) + (s[2][lane] + s[3][lane]);
  if (gridDim.x == 1)
    out[j] = T(t);
  else
    sums[int64_t(blockIdx.x) * n + j] = t;
}

// Sums over parts of partial[part, e], e < length: out (rows x cols) takes the
// first rows * cols, tail the rest.  A block takes 64 neighbouring elements; its
// 16 waves take every 16th part each and their sums are added in order.
constexpr int kJoinWaves = 16;
template <typename T>
__global__ __launch_bounds__(64 * kJoinWaves) void join_parts_kernel(const float* __restrict__ partial, int64_t parts,
                                                                     int64_t length, int64_t first, int64_t last,
                                                                     int64_t cols, int64_t size, T* __restrict__ out,
                                                                     int64_t out_ld, T* __restrict__ tail) {
  __shared__ float s[kJoinWaves][64];
  const int lane = threadIdx.x % 64, w = threadIdx.x / 64;
  for (int64_t b = first + int64_t(blockIdx.x) * 64; b < last; b += int64_t(gridDim.x) * 64) {
    const int64_t e = b + lane;
    float t = 0.0f;
    if (e < last) {
#pragma unroll 8
      for (int64_t p = w; p < parts; p += kJoinWaves) t += partial[p * length + e];
    }
    s[w][lane] = t;
    __syncthreads();
    if (w == 0 && e < last) {
      float sum = s[0][lane];
#pragma unroll
      for (int v = 1; v < kJoinWaves; ++v) sum += s[v][lane];
      if (e < size)
        out[e / cols * out_ld + e % cols] = T(sum);
      else
        tail[e - size] = T(sum);
    }
    __syncthreads();
  }
}

// partial [parts, rows * cols + more]: out (may be NULL) and tail (may be NULL)
template <typename T>
hipError_t join_parts(const float* partial, int64_t parts, int64_t rows, int64_t cols, void* out, int64_t ld,
                      hipStream_t s, int64_t more = 0, void* tail = nullptr) {
  const int64_t size = rows * cols, first = out ? 0 : size, last = tail ? size + more : size;
  if (last <= first) return hipSuccess;
  const int64_t blocks = std::min<int64_t>(ceil_div64(last - first, 64), 1 << 16);
  join_parts_kernel<T><<<uint32_t(blocks), 64 * kJoinWaves, 0, s>>>(
      partial, parts, size + more, first, last, cols, size, static_cast<T*>(out), ld, static_cast<T*>(tail));
  return hipGetLastError();
}

// y, dz or g_x from the parts of its sums: a block takes kJoinRows rows times 64
// columns, and for dz leaves its column sums.
template <typename T, Epilogue EPI>
__global__ __launch_bounds__(256) void join_rows_kernel(const GemmArgs g, const float* __restrict__ partial,
                                                        int64_t parts) {
  __shared__ float s[4][64];
  const int lane = threadIdx.x % 64, w = threadIdx.x / 64;
  const int64_t j = int64_t(blockIdx.x) * 64 + lane, r0 = int64_t(blockIdx.y) * kJoinRows;
  float sum = 0.0f;
  if (j < g.cols) {
    const float b = (EPI == EPI_FORWARD || EPI == EPI_DZ) && g.bias ? float(static_cast<const T*>(g.bias)[j]) : 0.0f;
    with_activation(g.act, [&](auto act) {
      for (int64_t r = r0 + w; r < min(g.rows, r0 + kJoinRows); r += 4) {
        float c = 0.0f;
#pragma unroll 4
        for (int64_t p = 0; p < parts; ++p) c += partial[(p * g.rows + r) * g.cols + j];
        const T* extra = static_cast<const T*>(g.extra) + r * g.extra_ld + j;
        if constexpr (EPI == EPI_FORWARD) {
          c = activate<decltype(act)::value>(c + b);
          if (g.extra) c += float(*extra);
        }
        if constexpr (EPI == EPI_DZ) {
          c = activate_grad<decltype(act)::value>(c + b, float(*extra));
          sum += c;
        }
        T* out = static_cast<T*>(g.out) + r * g.out_ld + j;
        if constexpr (EPI == EPI_DZ && sizeof(T) == 2) {
          if (g.out_low) {
            split_dz<T>(c, *out, out[g.out_low]);
            continue;
          }
        }
        *out = T(c);
      }
    });
  }
  if constexpr (EPI == EPI_DZ) {
    s[w][lane] = sum;
    __syncthreads();
    if (w == 0 && j < g.cols && g.sums)
      g.sums[int64_t(blockIdx.y) * g.cols + j] = (s[0][lane] + s[1][lane]) + (s[2][lane] + s[3][lane]);
  }
}

template <typename T, bool AKC, bool BKC, Epilogue EPI, bool PARTS>
hipError_t run_tiles(GemmArgs g, const Cut& c, hipStream_t s) {
  g.tiles_i = ceil_div64(g.rows, c.rows);
  g.tiles_j = ceil_div64(g.cols, c.cols);
  g.part = c.part;
  const dim3 grid(uint32_t(g.tiles_i * g.tiles_j), 1, uint32_t(EPI == EPI_PARTIAL ? c.parts : 1));
  if (c.rows == 64) {
    gemm_kernel<T, AKC, BKC, 2, 2, 2, 2, false, EPI, PARTS><<<grid, 256, 0, s>>>(g);
  } else if (c.cols == 32) {
    gemm_kernel<T, AKC, BKC, 2, 2, 4, 1, false, EPI, PARTS><<<grid, 256, 0, s>>>(g);
  } else if (c.rows == 32) {
    gemm_kernel<T, AKC, BKC, 2, 2, 1, 4, false, EPI, PARTS><<<grid, 256, 0, s>>>(g);
  } else if (c.rows == 128) {
    gemm_kernel<T, AKC, BKC, 4, 4, 2, 2, false, EPI, PARTS><<<grid, 256, 0, s>>>(g);
  } else {
    if constexpr (sizeof(T) == 2 && EPI != EPI_PARTIAL)
      gemm_kernel<T, AKC, BKC, 8, 4, 2, 4, true, EPI, PARTS><<<grid, 512, 0, s>>>(g);
    else
      return hipErrorInvalidValue;
  }
  return hipGetLastError();
}

// Tiles of 256 need 16-byte aligned rows, whole steps of k and, for lines
// across k, whole packs of rows.
template <typename T>
bool wide_operand(const void* p, int64_t ld, int64_t rows, bool kc) {
  return sizeof(T) == 2 && reinterpret_cast<uintptr_t>(p) % 16 == 0 && ld % 8 == 0 && (kc || rows % 8 == 0);
}

// The product with its epilogue; partial holds parts * rows * cols floats where
// it is cut.  *sum_parts: the column sums that EPI_DZ leaves.
template <typename T, bool AKC, bool BKC, Epilogue EPI, bool PARTS = false>
hipError_t product(GemmArgs g, int64_t most, float* partial, hipStream_t s, int64_t* sum_parts = nullptr) {
  if (g.rows <= 0 || g.cols <= 0) return hipSuccess;
  const bool wide = g.depth % 64 == 0 && wide_operand<T>(g.a, g.a_ld, g.rows, AKC) &&
                    wide_operand<T>(g.b, g.b_ld, g.cols, BKC);
  const Cut c = cut_product(g.rows, g.cols, g.depth, most, wide);
  if (sum_parts) *sum_parts = ceil_div64(g.rows, c.parts == 1 ? c.rows : kJoinRows);
  if (c.parts == 1) return run_tiles<T, AKC, BKC, EPI, PARTS>(g, c, s);
  GemmArgs p = g;
  p.out = partial;
  const hipError_t e = run_tiles<T, AKC, BKC, EPI_PARTIAL, PARTS>(p, c, s);
  if (e != hipSuccess) return e;
  if constexpr (EPI == EPI_STORE) {
    if (c.parts > kJoinParts) return join_parts<T>(partial, c.parts, g.rows, g.cols, g.out, g.out_ld, s);
  }
  const dim3 grid(uint32_t(ceil_div64(g.cols, 64)), uint32_t(ceil_div64(g.rows, kJoinRows)));
  join_rows_kernel<T, EPI><<<grid, 256, 0, s>>>(g, partial, c.parts);
  return hipGetLastError();
}

// A product of dz, which is in two parts where g.a_low says so.
template <typename T, bool AKC>
hipError_t dz_product(const GemmArgs& g, int64_t most, float* partial, hipStream_t s) {
  if constexpr (sizeof(T) == 2) {
    if (g.a_low) return product<T, AKC, false, EPI_STORE, true>(g, most, partial, s);
  }
  return product<T, AKC, false, EPI_STORE>(g, most, partial, s);
}

template <typename T>
GemmArgs layer_product(const LinearArgs& a) {  // x W^T
  GemmArgs g{};
  g.a = a.x;
  g.a_ld = a.x_ld;
  g.b = a.w;
  g.b_ld = a.w_ld;
  g.rows = a.m;
  g.cols = a.n;
  g.depth = a.k;
  g.act = a.act;
  g.bias = a.bias;
  return g;
}

}  // namespace

template <typename T>
hipError_t gemm_forward(const LinearArgs& a, hipStream_t s) {
  GemmArgs g = layer_product<T>(a);
  g.extra = a.residual;
  g.extra_ld = a.residual_ld;
  g.out = a.y;
  g.out_ld = a.y_ld;
  return product<T, true, true, EPI_FORWARD>(g, kJoinParts, static_cast<float*>(a.scratch), s);
}

template <typename T>
hipError_t gemm_backward(const LinearArgs& a, hipStream_t s) {
  const BackwardPlan p = backward_plan(a.m, a.k, a.n, kType<T>, a.act);
  char* base = static_cast<char*>(a.scratch);
  float* sums = reinterpret_cast<float*>(base + p.sums);
  float* partial = reinterpret_cast<float*>(base + p.partial);
  hipError_t e = hipSuccess;
  if constexpr (sizeof(T) == 2) {
    if (p.small) return small_backward<T>(a, reinterpret_cast<float*>(base + p.dz), s);
  }
  if (p.stream) {
    if ((e = stream_backward<T>(a, partial, s)) != hipSuccess || p.parts == 1) return e;
    return join_parts<T>(partial, p.parts, a.n, a.k, a.g_w, a.g_w_ld, s, a.n, a.g_bias);
  }
  const void* dz = a.dl;
  int64_t dz_ld = a.dl_ld, dz_low = 0, sum_parts = 0;
  bool bias_done = false;
  if (a.act != GART_ACT_NONE) {
    dz = base + p.dz;
    dz_ld = p.dz_ld;
    dz_low = p.dz_low;
    if (few_rows(a.m, a.k, a.n, sizeof(T))) {
      e = rows_dz<T>(a, base + p.dz, dz_ld, dz_low, s);
      bias_done = a.m > 0;
    } else {
      GemmArgs g = layer_product<T>(a);
      g.extra = a.dl;
      g.extra_ld = a.dl_ld;
      g.out = base + p.dz;
      g.out_ld = dz_ld;
      g.out_low = dz_low;
      g.sums = a.g_bias ? sums : nullptr;
      e = product<T, true, true, EPI_DZ>(g, kJoinParts, partial, s, &sum_parts);
    }
  } else if (a.g_bias && a.m > 0 && a.n > 0) {
    sum_parts = ceil_div64(a.m, kSumRows);
    column_sums_kernel<T><<<dim3(uint32_t(sum_parts), uint32_t(ceil_div64(a.n, 64))), 256, 0, s>>>(
        static_cast<const T*>(a.dl), a.dl_ld, a.m, a.n, sums, static_cast<T*>(a.g_bias));
    e = hipGetLastError();
    bias_done = sum_parts == 1;
  }
  if (e != hipSuccess) return e;
  if (a.g_bias && !bias_done && (e = join_parts<T>(sums, sum_parts, 1, a.n, a.g_bias, a.n, s)) != hipSuccess) return e;
  GemmArgs g{};
  g.a = dz;
  g.a_ld = dz_ld;
  g.a_low = dz_low;
  if (a.g_x) {
    g.b = a.w;
    g.b_ld = a.w_ld;
    g.rows = a.m;
    g.cols = a.k;
    g.depth = a.n;
    g.out = a.g_x;
    g.out_ld = a.g_x_ld;
    if ((e = dz_product<T, true>(g, kJoinParts, partial, s)) != hipSuccess) return e;
  }
  if (a.g_w) {
    g.b = a.x;
    g.b_ld = a.x_ld;
    g.rows = a.n;
    g.cols = a.k;
    g.depth = a.m;
    g.out = a.g_w;
    g.out_ld = a.g_w_ld;
    return dz_product<T, false>(g, kWeightParts, partial, s);
  }
  return hipSuccess;
}

}  // namespace gart
