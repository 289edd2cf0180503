// Linear layer y = act(x W^T + b) + residual and its gradient on the matrix cores.
//
// Products are C[i,j] = sum_k A(i,k) B(j,k) on 16x16 tiles, sums in float.
// B's tile is the matrix instruction's first operand, so a lane holds four
// consecutive j of one i and stores along rows.  An operand is either
// k-contiguous (x and W of the forward) or i-contiguous (the gradient's, whose
// sums run over rows): the first kind lies in LDS as rows of 128 bytes with
// their 16-byte pieces exchanged by row, the second as it comes from memory,
// and 16-bit fragments of it are read with the transposing LDS load.
#include <algorithm>

#include "blocks.h"

namespace gart {
namespace {

typedef float f32x4 __attribute__((ext_vector_type(4)));

template <typename T>
struct Mfma;

// 16 bits: 16x16x32, eight consecutive k a lane.
template <>
struct Mfma<bf16> {
  static __device__ __forceinline__ f32x4 run(Pack<bf16>::V a, Pack<bf16>::V b, f32x4 c) {
    return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0);
  }
};
template <>
struct Mfma<f16> {
  static __device__ __forceinline__ f32x4 run(Pack<f16>::V a, Pack<f16>::V b, f32x4 c) {
    return __builtin_amdgcn_mfma_f32_16x16x32_f16(a, b, c, 0, 0, 0);
  }
};
// float: four 16x16x4, one k a lane each.  Which k a lane holds is free as
// long as both operands agree, so it holds four consecutive ones, as one read.
template <>
struct Mfma<float> {
  static __device__ __forceinline__ f32x4 run(Pack<float>::V a, Pack<float>::V b, f32x4 c) {
#pragma unroll
    for (int t = 0; t < 4; ++t) c = __builtin_amdgcn_mfma_f32_16x16x4f32(a[t], b[t], c, 0, 0, 0);
    return c;
  }
};

// ---- activations -----------------------------------------------------------
// silu(z) = z g(z) and gelu(z) = z g(2 sqrt(2/pi) (z + 0.044715 z^3)) with the
// logistic function g(u) = 1 / (1 + exp(-u)).  Beyond |u| = 87 g is 0 or 1 in
// float and g' is 0.
constexpr float kGelu = 1.5957691216057308f;  // 2 sqrt(2 / pi)

struct Gate {
  float g, slope;  // g(u), g'(u)
};

__device__ __forceinline__ Gate gate(float u) {
  // exp(-u) = 2^h 2^l: h the rounded product, l what it lost and the low part
  // of log2(e), so that float results keep their last bits for large |u|
  const float c = fminf(fmaxf(-u, -87.0f), 87.0f);
  const float h = c * 1.44269504f;
  const float l = fmaf(c, 1.44269504f, -h) + c * 1.92596299e-8f;
  float e = __builtin_amdgcn_exp2f(h);
  e = fmaf(e, l * 0.693147181f, e);
  Gate r;
  r.g = __builtin_amdgcn_rcpf(1.0f + e);
  r.slope = e * r.g * r.g;
  if (u < -87.0f) r.g = 0.0f;
  if (fabsf(u) > 87.0f) r.slope = 0.0f;
  return r;
}

__device__ __forceinline__ float gate_argument(float z, gart_activation act) {
  return act == GART_ACT_GELU ? kGelu * fmaf(0.044715f * z * z, z, z) : z;
}

__device__ __forceinline__ float activate(float z, gart_activation act) {
  if (act == GART_ACT_NONE) return z;
  if (act == GART_ACT_RELU) return z < 0.0f ? 0.0f : z;  // a NaN stays
  const float g = gate(gate_argument(z, act)).g;
  return g == 0.0f ? 0.0f : z * g;  // not inf * 0 at -infinity
}

// dl times act'(z)
__device__ __forceinline__ float activate_grad(float z, float dl, gart_activation act) {
  if (act == GART_ACT_NONE) return dl;
  if (act == GART_ACT_RELU) return z <= 0.0f ? 0.0f : dl;
  const Gate t = gate(gate_argument(z, act));
  const float du = act == GART_ACT_GELU ? kGelu * fmaf(0.134145f * z, z, 1.0f) : 1.0f;
  return dl * (t.slope == 0.0f && z == z ? t.g : fmaf(z * t.slope, du, t.g));
}

// ---- tiles -------------------------------------------------------------------
constexpr int kLine = 128;  // bytes of k per step

template <typename T>
constexpr int kStep = kLine / int(sizeof(T));  // k per step

// One operand's tile of ROWS rows (i) and kStep columns (k) in LDS.  PERM: the
// rows a fragment takes are the output's j, paired up below.
template <typename T, bool KC, int ROWS, int THREADS, bool PERM>
struct Tile {
  static constexpr int V = Pack<T>::N;
  static constexpr int PITCH = KC ? kStep<T> : ROWS + 64 / int(sizeof(T)) / (sizeof(T) == 4 ? 4 : 2);
  static constexpr int ELEMS = KC ? ROWS * PITCH : kStep<T> * PITCH;
  static constexpr int LINE_PACKS = KC ? kStep<T> / V : ROWS / V;  // packs per line in memory
  static constexpr int LINES = KC ? ROWS : kStep<T>;
  static constexpr int PACKS = LINES * LINE_PACKS;
  static constexpr int PER_THREAD = (PACKS + THREADS - 1) / THREADS;

  // 16 bits: tiles 2q and 2q+1 together hold 32 j, eight consecutive ones a
  // lane.  float: a lane's four consecutive j are 16 bytes already.
  static __device__ __forceinline__ int frag_row(int tile, int r) {
    if (PERM && sizeof(T) == 2) return 32 * (tile / 2) + 8 * (r / 4) + 4 * (tile % 2) + r % 4;
    return 16 * tile + r;
  }
  // exchange of a row's 16-byte pieces: distinct for any eight lanes that read together
  static __device__ __forceinline__ int swizzle(int row) {
    return PERM && sizeof(T) == 2 ? (row & 3) | ((row >> 1) & 4) : row & 7;
  }

  Pack<T> reg[PER_THREAD];

  // rows x ks elements are there; i0, k0: where the tile begins
  __device__ __forceinline__ void load(const T* __restrict__ p, int64_t ld, int64_t i0, int64_t rows, int64_t k0,
                                       int64_t ks, int tid) {
#pragma unroll
    for (int u = 0; u < PER_THREAD; ++u) {
      const int c = u * THREADS + tid;
      const int line = c / LINE_PACKS, at = (c % LINE_PACKS) * V;
      const int64_t l = (KC ? i0 : k0) + line, o = (KC ? k0 : i0) + at;
      const int64_t lines = KC ? rows : ks, length = KC ? ks : rows;
      reg[u].v = T(0.0f);
      if ((PACKS % THREADS == 0 || c < PACKS) && l < lines && o < length)
        reg[u] = load_some(p + l * ld + o, int(min(int64_t(V), length - o)));
    }
  }
  __device__ __forceinline__ void store(T* lds, int tid) const {
#pragma unroll
    for (int u = 0; u < PER_THREAD; ++u) {
      const int c = u * THREADS + tid;
      if (PACKS % THREADS != 0 && c >= PACKS) continue;
      const int line = c / LINE_PACKS;
      int piece = c % LINE_PACKS;
      if (KC) piece ^= swizzle(line);
      *reinterpret_cast<typename Pack<T>::V*>(lds + line * PITCH + piece * V) = reg[u].v;
    }
  }
  // fragment of 16 rows at tile `tile`, k step `s` (32 k of 16 bits, 16 of floats)
  static __device__ __forceinline__ typename Pack<T>::V fragment(const T* lds, int tile, int s, int lane) {
    const int r = lane % 16, g = lane / 16;
    if constexpr (KC) {
      const int row = frag_row(tile, r);
      return *reinterpret_cast<const typename Pack<T>::V*>(lds + row * PITCH + ((4 * s + g) ^ swizzle(row)) * V);
    } else if constexpr (sizeof(T) == 4) {
      const T* q = lds + (16 * s + 4 * g) * PITCH + frag_row(tile, r);
      typename Pack<T>::V v;
#pragma unroll
      for (int t = 0; t < 4; ++t) v[t] = q[t * PITCH];
      return v;
    } else {
      // the lanes of a group of 16 name four k times 16 columns, four a lane;
      // each receives the four k of its column
      typedef short s16x4 __attribute__((ext_vector_type(4)));
      typedef __attribute__((address_space(3))) s16x4* lds_ptr;
      const T* q = lds + (32 * s + 8 * g + r / 4) * PITCH + frag_row(tile, 4 * (r % 4));
      const s16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_ptr)(q));
      const s16x4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_ptr)(q + 4 * PITCH));
      typename Pack<T>::V v;
      __builtin_memcpy(&v, &lo, 8);
      __builtin_memcpy(reinterpret_cast<char*>(&v) + 8, &hi, 8);
      return v;
    }
  }
};

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
  int64_t rows, cols, depth;  // of C, and the length of the sums
  int64_t part;               // length of one part of the sums (EPI_PARTIAL: blockIdx.z)
  int64_t tiles_i, tiles_j;
  gart_activation act;
  const void *bias, *extra;  // extra: residual or dl
  int64_t extra_ld;
  void* out;
  int64_t out_ld;
  float* sums;  // EPI_DZ: [tiles_i, cols] column sums, or NULL
};

// Blocks are dealt to the eight XCDs in turn; each XCD gets a contiguous run of
// tiles, which share rows of A in its L2.
__device__ __forceinline__ int64_t xcd_tile(int64_t b, int64_t total) {
  const int64_t q = total / 8, r = total % 8, x = b % 8;
  return x * q + min(x, r) + b / 8;
}

template <typename T, bool AKC, bool BKC, int TI, int TJ, int WI, int WJ, Epilogue EPI>
__global__ __launch_bounds__(64 * WI * WJ) void gemm_kernel(const GemmArgs g) {
  constexpr int THREADS = 64 * WI * WJ;
  using TA = Tile<T, AKC, 16 * TI * WI, THREADS, false>;
  using TB = Tile<T, BKC, 16 * TJ * WJ, THREADS, true>;
  constexpr int BI = 16 * TI * WI, BJ = 16 * TJ * WJ, V = Pack<T>::N;
  __shared__ __attribute__((aligned(16))) T lds[2][TA::ELEMS + TB::ELEMS];
  __shared__ float s_sum[EPI == EPI_DZ ? WI : 1][EPI == EPI_DZ ? BJ : 1];

  const int tid = threadIdx.x, lane = tid % 64, wave = tid / 64;
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

  TA ta;
  TB tb;
  ta.load(pa, g.a_ld, i0, g.rows, k0, k1, tid);
  tb.load(pb, g.b_ld, j0, g.cols, k0, k1, tid);
  int buf = 0;
  for (int64_t k = k0; k < k1; k += kStep<T>) {
    T* la = lds[buf];
    T* lb = la + TA::ELEMS;
    ta.store(la, tid);
    tb.store(lb, tid);
    __syncthreads();  // also: the other buffer's readers are past it once all threads are here
    if (k + kStep<T> < k1) {
      ta.load(pa, g.a_ld, i0, g.rows, k + kStep<T>, k1, tid);
      tb.load(pb, g.b_ld, j0, g.cols, k + kStep<T>, k1, tid);
    }
#pragma unroll
    for (int s = 0; s < 2; ++s) {
      typename Pack<T>::V fa[TI], fb[TJ];
#pragma unroll
      for (int i = 0; i < TI; ++i) fa[i] = TA::fragment(la, wi * TI + i, s, lane);
#pragma unroll
      for (int j = 0; j < TJ; ++j) fb[j] = TB::fragment(lb, wj * TJ + j, s, lane);
#pragma unroll
      for (int i = 0; i < TI; ++i)
#pragma unroll
        for (int j = 0; j < TJ; ++j) acc[i][j] = Mfma<T>::run(fb[j], fa[i], acc[i][j]);
    }
    buf ^= 1;
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
      for (int e = 0; e < V; ++e) c[e] = acc[i][jq * JQ + e / 4][e % 4] + b[e];
      if constexpr (EPI == EPI_PARTIAL) {
        float* out = static_cast<float*>(g.out) + (int64_t(blockIdx.z) * g.rows + row) * g.out_ld + j;
#pragma unroll
        for (int e = 0; e < V; ++e)
          if (e < count) out[e] = c[e];
      } else {
        if constexpr (EPI == EPI_FORWARD) {
#pragma unroll
          for (int e = 0; e < V; ++e) c[e] = activate(c[e], g.act);
        }
        if (EPI == EPI_DZ || (EPI == EPI_FORWARD && g.extra)) {
          const Pack<T> p = load_some(static_cast<const T*>(g.extra) + row * g.extra_ld + j, count);
#pragma unroll
          for (int e = 0; e < V; ++e) {
            if constexpr (EPI == EPI_DZ) {
              c[e] = e < count ? activate_grad(c[e], float(p.v[e]), g.act) : 0.0f;
              sum[e] += c[e];
            } else {
              c[e] += float(p.v[e]);
            }
          }
        }
        Pack<T> o;
#pragma unroll
        for (int e = 0; e < V; ++e) o.v[e] = T(c[e]);
        store_some(static_cast<T*>(g.out) + row * g.out_ld + j, o, count);
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

// Column sums of m rows, one part of kSumRows rows a block: sums[part, n].
constexpr int kSumRows = 256;
template <typename T>
__global__ __launch_bounds__(256) void column_sums_kernel(const T* __restrict__ p, int64_t ld, int64_t m, int64_t n,
                                                          float* __restrict__ sums) {
  __shared__ float s[4][64];
  const int lane = threadIdx.x % 64, w = threadIdx.x / 64;
  const int64_t j = int64_t(blockIdx.y) * 64 + lane, r0 = int64_t(blockIdx.x) * kSumRows;
  float t = 0.0f;
  if (j < n)
    for (int64_t r = r0 + w; r < min(m, r0 + kSumRows); r += 4) t += float(p[r * ld + j]);
  s[w][lane] = t;
  __syncthreads();
  if (w == 0 && j < n) sums[int64_t(blockIdx.x) * n + j] = (s[0][lane] + s[1][lane]) + (s[2][lane] + s[3][lane]);
}

// out[i, j] = sum over parts of partial[part, i, j], in order of the parts
template <typename T>
__global__ __launch_bounds__(256) void join_parts_kernel(const float* __restrict__ partial, int64_t parts,
                                                         int64_t rows, int64_t cols, T* __restrict__ out,
                                                         int64_t out_ld) {
  const int64_t total = rows * cols;
  for (int64_t e = int64_t(blockIdx.x) * 256 + threadIdx.x; e < total; e += int64_t(gridDim.x) * 256) {
    float t = 0.0f;
    for (int64_t p = 0; p < parts; ++p) t += partial[p * total + e];
    out[e / cols * out_ld + e % cols] = T(t);
  }
}

template <typename T>
hipError_t join_parts(const float* partial, int64_t parts, int64_t rows, int64_t cols, void* out, int64_t ld,
                      hipStream_t s) {
  if (rows * cols <= 0) return hipSuccess;
  const int64_t blocks = std::min<int64_t>(ceil_div64(rows * cols, 256), 1 << 16);
  join_parts_kernel<T><<<uint32_t(blocks), 256, 0, s>>>(partial, parts, rows, cols, static_cast<T*>(out), ld);
  return hipGetLastError();
}

constexpr int kTile = 128;                       // rows and columns of C per block
constexpr int64_t kMaxTiles = int64_t(1) << 23;  // blocks of a launch

template <typename T, bool AKC, bool BKC, Epilogue EPI>
hipError_t gemm(GemmArgs g, hipStream_t s) {
  if (g.rows <= 0 || g.cols <= 0) return hipSuccess;
  g.tiles_i = ceil_div64(g.rows, kTile);
  g.tiles_j = ceil_div64(g.cols, kTile);
  const int64_t parts = EPI == EPI_PARTIAL ? ceil_div64(g.depth, g.part) : 1;
  gemm_kernel<T, AKC, BKC, 4, 4, 2, 2, EPI>
      <<<dim3(uint32_t(g.tiles_i * g.tiles_j), 1, uint32_t(parts)), 256, 0, s>>>(g);
  return hipGetLastError();
}

// ---- gradient ----------------------------------------------------------------
struct BackwardPlan {
  int64_t dz_ld, part, parts, sum_parts;
  size_t dz, partial, sums, total;
};

BackwardPlan backward_plan(int64_t m, int64_t k, int64_t n, size_t es, gart_activation act) {
  BackwardPlan p{};
  size_t off = 0;
  auto take = [&](size_t bytes) {
    const size_t o = off;
    off += (bytes + 255) & ~size_t(255);
    return o;
  };
  p.dz_ld = (n + 7) / 8 * 8;
  p.dz = take(act == GART_ACT_NONE ? 0 : size_t(m) * size_t(p.dz_ld) * es);
  // the weight's gradient sums over the rows: enough parts to fill the card
  const int64_t tiles = std::max<int64_t>(1, ceil_div64(n, kTile) * ceil_div64(k, kTile));
  const int64_t want = std::max<int64_t>(1, 512 / tiles);
  p.part = std::max<int64_t>(256, ceil_div64(ceil_div64(std::max<int64_t>(m, 1), want), 256) * 256);
  p.parts = ceil_div64(m, p.part);
  p.partial = take(size_t(p.parts) * size_t(n) * size_t(k) * 4);
  p.sum_parts = act == GART_ACT_NONE ? ceil_div64(m, kSumRows) : ceil_div64(m, kTile);
  p.sums = take(size_t(p.sum_parts) * size_t(n) * 4);
  p.total = off;
  return p;
}

template <typename T>
hipError_t forward(const LinearArgs& a, hipStream_t s) {
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
  g.extra = a.residual;
  g.extra_ld = a.residual_ld;
  g.out = a.y;
  g.out_ld = a.y_ld;
  return gemm<T, true, true, EPI_FORWARD>(g, s);
}

template <typename T>
hipError_t backward(const LinearArgs& a, hipStream_t s) {
  const BackwardPlan p = backward_plan(a.m, a.k, a.n, sizeof(T), a.act);
  char* base = static_cast<char*>(a.scratch);
  const void* dz = a.dl;
  int64_t dz_ld = a.dl_ld;
  float* sums = reinterpret_cast<float*>(base + p.sums);
  hipError_t e;
  if (a.act != GART_ACT_NONE) {
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
    g.extra = a.dl;
    g.extra_ld = a.dl_ld;
    g.out = base + p.dz;
    g.out_ld = p.dz_ld;
    g.sums = a.g_bias ? sums : nullptr;
    if ((e = gemm<T, true, true, EPI_DZ>(g, s)) != hipSuccess) return e;
    dz = base + p.dz;
    dz_ld = p.dz_ld;
  } else if (a.g_bias && a.m > 0 && a.n > 0) {
    column_sums_kernel<T><<<dim3(uint32_t(p.sum_parts), uint32_t(ceil_div64(a.n, 64))), 256, 0, s>>>(
        static_cast<const T*>(a.dl), a.dl_ld, a.m, a.n, sums);
    if ((e = hipGetLastError()) != hipSuccess) return e;
  }
  if (a.g_bias)
    if ((e = join_parts<T>(sums, p.sum_parts, 1, a.n, a.g_bias, a.n, s)) != hipSuccess) return e;
  if (a.g_x) {
    GemmArgs g{};
    g.a = dz;
    g.a_ld = dz_ld;
    g.b = a.w;
    g.b_ld = a.w_ld;
    g.rows = a.m;
    g.cols = a.k;
    g.depth = a.n;
    g.out = a.g_x;
    g.out_ld = a.g_x_ld;
    if ((e = gemm<T, true, false, EPI_STORE>(g, s)) != hipSuccess) return e;
  }
  if (a.g_w) {
    GemmArgs g{};
    g.a = dz;
    g.a_ld = dz_ld;
    g.b = a.x;
    g.b_ld = a.x_ld;
    g.rows = a.n;
    g.cols = a.k;
    g.depth = a.m;
    g.part = p.part;
    g.out = base + p.partial;
    g.out_ld = a.k;
    if (a.m > 0 && (e = gemm<T, false, false, EPI_PARTIAL>(g, s)) != hipSuccess) return e;
    return join_parts<T>(reinterpret_cast<float*>(base + p.partial), p.parts, a.n, a.k, a.g_w, a.g_w_ld, s);
  }
  return hipSuccess;
}

}  // namespace

int64_t linear_scratch_bytes(int64_t m, int64_t, int64_t n, gart_dtype) {
  return ceil_div64(m, kTile) * ceil_div64(n, kTile) > kMaxTiles ? -1 : 0;
}

int64_t linear_backward_scratch_bytes(int64_t m, int64_t k, int64_t n, gart_dtype t, gart_activation act) {
  const int64_t mt = ceil_div64(m, kTile), nt = ceil_div64(n, kTile), kt = ceil_div64(k, kTile);
  if (mt * nt > kMaxTiles || mt * kt > kMaxTiles || nt * kt > kMaxTiles) return -1;
  return int64_t(backward_plan(m, k, n, dtype_bytes(t), act).total);
}

hipError_t launch_linear(const LinearArgs& a, gart_dtype t, hipStream_t s) {
  if (t == GART_DTYPE_F32) return forward<float>(a, s);
  if (t == GART_DTYPE_BF16) return forward<bf16>(a, s);
  return forward<f16>(a, s);
}

hipError_t launch_linear_backward(const LinearArgs& a, gart_dtype t, hipStream_t s) {
  if (t == GART_DTYPE_F32) return backward<float>(a, s);
  if (t == GART_DTYPE_BF16) return backward<bf16>(a, s);
  return backward<f16>(a, s);
}

}  // namespace gart
