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

#include "linear.h"

namespace gart {
namespace {

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
  // fragment of 16 rows at tile `tile`, step `s` of the line's two
  static __device__ __forceinline__ typename Pack<T>::V fragment(const T* lds, int tile, int s, int lane) {
    if constexpr (KC) {
      const int r = lane % 16, g = lane / 16, row = PERM ? paired_row<T>(tile, r) : 16 * tile + r;
      return fragment_of_row(lds, PITCH, row, 0, (4 * s + g) ^ swizzle(row));
    } else {
      return fragment_of_columns<T, PERM>(lds, PITCH, tile, kDepth<T> * s, lane);
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

// out[i, j] = sum over parts of partial[part, i, j].  A block takes 64
// neighbouring elements; its 16 waves take every 16th part each and their sums
// are added in order.
constexpr int kJoinWaves = 16;
template <typename T>
__global__ __launch_bounds__(64 * kJoinWaves) void join_parts_kernel(const float* __restrict__ partial, int64_t parts,
                                                                     int64_t rows, int64_t cols, T* __restrict__ out,
                                                                     int64_t out_ld) {
  __shared__ float s[kJoinWaves][64];
  const int lane = threadIdx.x % 64, w = threadIdx.x / 64;
  const int64_t total = rows * cols;
  for (int64_t b = int64_t(blockIdx.x) * 64; b < total; b += int64_t(gridDim.x) * 64) {
    const int64_t e = b + lane;
    float t = 0.0f;
    if (e < total) {
#pragma unroll 4
      for (int64_t p = w; p < parts; p += kJoinWaves) t += partial[p * total + e];
    }
    s[w][lane] = t;
    __syncthreads();
    if (w == 0 && e < total) {
      float sum = s[0][lane];
#pragma unroll
      for (int v = 1; v < kJoinWaves; ++v) sum += s[v][lane];
      out[e / cols * out_ld + e % cols] = T(sum);
    }
    __syncthreads();
  }
}

template <typename T>
hipError_t join_parts(const float* partial, int64_t parts, int64_t rows, int64_t cols, void* out, int64_t ld,
                      hipStream_t s) {
  if (rows * cols <= 0) return hipSuccess;
  const int64_t blocks = std::min<int64_t>(ceil_div64(rows * cols, 64), 1 << 16);
  join_parts_kernel<T><<<uint32_t(blocks), 64 * kJoinWaves, 0, s>>>(partial, parts, rows, cols, static_cast<T*>(out), ld);
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
  bool stream;
  int64_t dz_ld, part, parts, sum_parts;
  size_t dz, partial, sums, total;
};

BackwardPlan backward_plan(int64_t m, int64_t k, int64_t n, gart_dtype t, gart_activation act) {
  BackwardPlan p{};
  const size_t es = dtype_bytes(t);
  size_t off = 0;
  auto take = [&](size_t bytes) {
    const size_t o = off;
    off += (bytes + 255) & ~size_t(255);
    return o;
  };
  p.parts = p.sum_parts = stream_backward_parts(m, k, n, t);
  if (p.parts > 0) {
    p.stream = true;
    p.partial = take(size_t(p.parts) * size_t(n) * size_t(k) * 4);
    p.sums = take(size_t(p.parts) * size_t(n) * 4);
    p.total = off;
    return p;
  }
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
hipError_t forward(const LinearArgs& a, gart_dtype t, hipStream_t s) {
  if (stream_forward_fits(a.k, a.n, t)) return launch_stream_forward(a, t, s);
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
hipError_t backward(const LinearArgs& a, gart_dtype t, hipStream_t s) {
  const BackwardPlan p = backward_plan(a.m, a.k, a.n, t, a.act);
  char* base = static_cast<char*>(a.scratch);
  const void* dz = a.dl;
  int64_t dz_ld = a.dl_ld;
  float* sums = reinterpret_cast<float*>(base + p.sums);
  float* partial = reinterpret_cast<float*>(base + p.partial);
  hipError_t e;
  if (p.stream) {
    if ((e = launch_stream_backward(a, partial, sums, t, s)) != hipSuccess) return e;
    if (a.g_w && (e = join_parts<T>(partial, p.parts, a.n, a.k, a.g_w, a.g_w_ld, s)) != hipSuccess) return e;
    return a.g_bias ? join_parts<T>(sums, p.parts, 1, a.n, a.g_bias, a.n, s) : hipSuccess;
  }
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
    g.out = partial;
    g.out_ld = a.k;
    if (a.m > 0 && (e = gemm<T, false, false, EPI_PARTIAL>(g, s)) != hipSuccess) return e;
    return join_parts<T>(partial, p.parts, a.n, a.k, a.g_w, a.g_w_ld, s);
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
  return int64_t(backward_plan(m, k, n, t, act).total);
}

hipError_t launch_linear(const LinearArgs& a, gart_dtype t, hipStream_t s) {
  if (t == GART_DTYPE_F32) return forward<float>(a, t, s);
  if (t == GART_DTYPE_BF16) return forward<bf16>(a, t, s);
  return forward<f16>(a, t, s);
}

hipError_t launch_linear_backward(const LinearArgs& a, gart_dtype t, hipStream_t s) {
  if (t == GART_DTYPE_F32) return backward<float>(a, t, s);
  if (t == GART_DTYPE_BF16) return backward<bf16>(a, t, s);
  return backward<f16>(a, t, s);
}

}  // namespace gart
