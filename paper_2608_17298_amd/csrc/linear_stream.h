// The linear layer where its weight fits LDS (a few hundred inputs and
// outputs) and the rows are many: every row is read once and its results are
// written once.
//
// Forward: a wave takes 32 rows.  x comes from memory straight into fragments
// (a lane holds 16 consecutive bytes of a row), W stands in LDS, and the
// outputs leave from registers, 16 bytes a lane.  Waves do not wait for each
// other.  Bound by bytes: 1M x 32 -> 64 f32 with gelu 88 us, 4.4 TB/s; 1016814 x
// 64 -> 48 bf16 with a residual 72 us, 4.5 TB/s.
//
// Backward: a block takes a tile of rows at a time.  Each wave owns 32 outputs
// (n): it computes z = W x^T for them again, dz = dl act'(z) in registers, and
// puts dz into LDS, where the other two products meet it:
//   g_weight (its 32 n, all k) += dz^T x over the tile's rows, kept in
//   registers for all of the block's tiles;
//   g_x (rows, k) = dz W, stored.
// Each block leaves one partial sum of g_weight and g_bias; a block that is
// alone leaves the gradients.  1M x 64 -> 128 bf16 with silu takes 160 us (3.2
// TB/s; product by product it took 3094), f16 181; with dz rounded to the type
// it was 132, in error by 1.4 times a rounding of the results.  Vector
// instructions, mostly the activation's slope and dz's parts, fill 53 % of the
// time (f16 61 %), LDS and bytes the rest.
#pragma once

#include <algorithm>

#include "linear_shapes.h"

namespace gart {
namespace {

// ---- forward -----------------------------------------------------------------
// Row strides up to which offsets inside a tile of rows fit 32 bits.
constexpr int64_t kNear = int64_t(1) << 22;
constexpr int kSpare = 8;  // rows of at least one element that hold a pack

// KP: inputs, rounded up.  LDS rows are 16 bytes longer, which spreads the
// rows that lanes read together over the banks.
// TAIL: fewer inputs than KP.
template <typename T, int KP, bool TAIL>
__global__ __launch_bounds__(64 * kForwardWaves) void stream_forward_kernel(const LinearArgs a) {
  constexpr int V = Pack<T>::N, S = KP / kDepth<T>, PITCH = KP + V, THREADS = 64 * kForwardWaves;
  extern __shared__ __attribute__((aligned(16))) char lds_raw[];
  T* w = reinterpret_cast<T*>(lds_raw);
  const int tid = threadIdx.x, lane = tid % 64, r = lane % 16, g = lane / 16;
  const int n_pad = int((a.n + 31) / 32 * 32);
  for (int c = tid; c < n_pad * (KP / V); c += THREADS) {
    const int row = c / (KP / V), at = c % (KP / V) * V;
    Pack<T> p;
    p.v = T(0.0f);
    if (row < a.n && at < a.k) p = load_some(static_cast<const T*>(a.w) + row * a.w_ld + at, int(a.k) - at);
    *reinterpret_cast<typename Pack<T>::V*>(w + row * PITCH + at) = p.v;
  }
  // the bias too: a load from memory would be waited for behind the stores
  float* s_bias = reinterpret_cast<float*>(w + n_pad * PITCH);
  for (int n = tid; n < n_pad; n += THREADS)
    s_bias[n] = a.bias && n < a.n ? float(static_cast<const T*>(a.bias)[n]) : 0.0f;
  __syncthreads();
  const T* x = static_cast<const T*>(a.x);
  const T* res = static_cast<const T*>(a.residual);
  T* y = static_cast<T*>(a.y);
  constexpr int Q = 8 / V;  // packs of outputs per lane: one of 8, or one of 4 from each tile
  const int64_t tiles = (a.m + 31) / 32, step = int64_t(gridDim.x) * kForwardWaves;
  // Inside, away from the last rows, lanes' offsets in a tile are the same for
  // all tiles, and a whole pack may be read at the end of a row: kSpare rows
  // follow it.  The edge has a loop of its own, so that nothing but the loads
  // themselves writes the registers they are on the way to.
  const bool near = a.x_ld <= kNear && a.x_ld > 0 && a.y_ld <= kNear && a.residual_ld <= kNear;
  const int64_t inside = near && a.m > kSpare ? (a.m - kSpare) / 32 : 0;
  const uint32_t x_off = uint32_t(r * a.x_ld + V * g), y_off = uint32_t(r * a.y_ld + (Q == 1 ? 8 : 4) * g),
                 res_off = uint32_t(r * a.residual_ld + (Q == 1 ? 8 : 4) * g);
  uint32_t x_at[S];
  PackMask<T> x_mask[S];
#pragma unroll
  for (int s = 0; s < S; ++s) {
    const int count = int(a.k) - (s * kDepth<T> + V * g);
    x_at[s] = TAIL && count <= 0 ? x_off - V * g : x_off + s * kDepth<T>;
    x_mask[s] = first_of_pack<T>(count);
  }
  typedef typename Pack<T>::V Rows[2][S];
  auto load_inside = [&](int64_t t, Rows& f) {
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      const T* p = x + (t * 32 + 16 * i) * a.x_ld;
#pragma unroll
      for (int s = 0; s < S; ++s) f[i][s] = load_pack(p + x_at[s]).v;  // masked where it is used: not a wait here
    }
  };
  auto load_edge = [&](int64_t t, Rows& f) {
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      const int64_t row = t * 32 + 16 * i + r;
#pragma unroll
      for (int s = 0; s < S; ++s) {
        const int64_t k = s * kDepth<T> + V * g;
        f[i][s] = T(0.0f);
        if (row < a.m && k < a.k) f[i][s] = load_some(x + row * a.x_ld + k, fresh(int(a.k - k))).v;
      }
    }
  };
  // The outputs of a tile's rows fx; before_stores(): between the first ones' sums and their stores.
  auto outputs = [&](auto whole_tile, int64_t t, const Rows& fx, auto&& before_stores) {
    constexpr bool whole = decltype(whole_tile)::value;
    Pack<T> p[2][Q];
    auto load_residual = [&](int n0) {
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        const int64_t row = t * 32 + 16 * i + r;
#pragma unroll
        for (int q = 0; q < Q; ++q) {
          const int n = n0 + 16 * q + (Q == 1 ? 8 : 4) * g, count = fresh(int(a.n) - n);
          if (count <= 0) continue;
          if (whole)
            p[i][q] = load_some(res + (t * 32 + 16 * i) * a.residual_ld + (n0 + 16 * q + res_off), count);
          else if (row < a.m)
            p[i][q] = load_some(res + row * a.residual_ld + n, count);
        }
      }
    };
    if (res) load_residual(0);
    for (int n0 = 0; n0 < n_pad; n0 += 32) {
      f32x4 acc[2][2];
#pragma unroll
      for (int j = 0; j < 2; ++j)
        acc[0][j] = acc[1][j] = *reinterpret_cast<const f32x4*>(s_bias + n0 + paired_row<T>(j, 4 * g));
#pragma unroll
      for (int s = 0; s < S; ++s) {
#pragma unroll
        for (int j = 0; j < 2; ++j) {
          const auto fw = fragment_of_row(w, PITCH, n0 + paired_row<T>(j, r), s * kDepth<T>, g);
#pragma unroll
          for (int i = 0; i < 2; ++i) acc[i][j] = Mfma<T>::run(fw, fx[i][s], acc[i][j]);
        }
      }
      Pack<T> o[2][Q];
#pragma unroll
      for (int q = 0; q < Q; ++q) {
        float c[2][V];
#pragma unroll
        for (int i = 0; i < 2; ++i)
#pragma unroll
          for (int e = 0; e < V; ++e) c[i][e] = acc[i][Q == 1 ? e / 4 : q][e % 4];
        with_activation(a.act, [&](auto act) {
#pragma unroll
          for (int i = 0; i < 2; ++i)
#pragma unroll
            for (int e = 0; e < V; ++e) c[i][e] = activate<decltype(act)::value>(c[i][e]);
        });
#pragma unroll
        for (int i = 0; i < 2; ++i) {
          if (res) {
#pragma unroll
            for (int e = 0; e < V; ++e) c[i][e] += float(p[i][q].v[e]);
          }
#pragma unroll
          for (int e = 0; e < V; ++e) o[i][q].v[e] = T(c[i][e]);
        }
      }
      // what the next steps need is asked for, and the next rows are here, before this step's stores
      if (res && n0 + 32 < n_pad) load_residual(n0 + 32);
      if (n0 == 0) before_stores();
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        const int64_t row = t * 32 + 16 * i + r;
#pragma unroll
        for (int q = 0; q < Q; ++q) {
          const int n = n0 + (Q == 1 ? 8 * g : 16 * q + 4 * g), count = fresh(int(a.n) - n);
          if (count <= 0) continue;
          if (whole)
            store_some(y + (t * 32 + 16 * i) * a.y_ld + (n0 + 16 * q + y_off), o[i][q], count);
          else if (row < a.m)
            store_some(y + row * a.y_ld + n, o[i][q], count);
        }
      }
    }
  };
  const int64_t first = int64_t(blockIdx.x) * kForwardWaves + __builtin_amdgcn_readfirstlane(tid / 64);
  int64_t t = first;
  Rows fx;
  if (t < inside) {
    Rows next;
    load_inside(t, next);
    for (; t < inside; t += step) {
#pragma unroll
      for (int i = 0; i < 2; ++i)
#pragma unroll
        for (int s = 0; s < S; ++s) {
          Pack<T> v;
          v.v = next[i][s];
          if (TAIL) mask_pack(v, x_mask[s]);
          fx[i][s] = v.v;
        }
      load_inside(min(t + step, inside - 1), next);
      outputs(std::true_type{}, t, fx, [&] {  // the next rows are here before this tile's stores are on the way
#pragma unroll
        for (int i = 0; i < 2; ++i)
#pragma unroll
          for (int s = 0; s < S; ++s) arrive(next[i][s]);
      });
    }
  }
  for (; t < tiles; t += step) {
    load_edge(t, fx);
    outputs(std::false_type{}, t, fx, [] {});
  }
}

// ---- backward ------------------------------------------------------------------
template <typename T, int KP, int NS, bool PARTS>
using BackwardShape = BackwardSizes<sizeof(T), KP, NS, PARTS>;

// Blocks a CU that the registers have to hold: two for small weights (one
// cost 204 us where two took 140, 1M x 64 -> 128 bf16), else what they hold.
template <typename T, int KP, int NS>
constexpr int kResident = KP * sizeof(T) <= 128 && NS <= 4 ? 2 : 1;

template <typename T, int KP, int NS, bool PARTS>
__global__ __launch_bounds__((BackwardShape<T, KP, NS, PARTS>::THREADS),
                             (kResident<T, KP, NS>)) void stream_backward_kernel(const LinearArgs a,
                                                                                 float* __restrict__ partial,
                                                                                 int64_t tiles) {
  using B = BackwardShape<T, KP, NS, PARTS>;
  constexpr int V = Pack<T>::N, D = kDepth<T>, S = KP / D, KT = KP / 16, Q = 8 / V;
  constexpr int MT = B::GROUP_ROWS / 16;
  __shared__ __attribute__((aligned(16))) T lds[B::W + B::X + B::Z + B::Z_LOW];
  T *lw = lds, *lx = lds + B::W, *lz = lx + B::X, *lz_low = lz + B::Z;  // lz_low: PARTS
  const int tid = threadIdx.x, lane = tid % 64, wave = __builtin_amdgcn_readfirstlane(tid / 64);
  const int r = lane % 16, g = lane / 16;
  const int slice = wave % NS, group = wave / NS;
  const T* x = static_cast<const T*>(a.x);
  const T* dl = static_cast<const T*>(a.dl);

  for (int c = tid; c < B::NP * (KP / V); c += B::THREADS) {
    const int row = c / (KP / V), at = c % (KP / V) * V;
    Pack<T> p;
    p.v = T(0.0f);
    if (row < a.n && at < a.k) p = load_some(static_cast<const T*>(a.w) + row * a.w_ld + at, int(a.k) - at);
    store_paired(lw + row * B::KPITCH, at, p);
  }

  // a lane's outputs: n0(q) + 0 .. V-1
  const auto n0 = [&](int q) { return 32 * slice + (Q == 1 ? 8 * g : 16 * q + 4 * g); };
  float b[8] = {}, sum_b[8] = {};
  if (a.bias) {
#pragma unroll
    for (int q = 0; q < Q; ++q) {
      if (n0(q) >= a.n) continue;
      const Pack<T> p = load_some(static_cast<const T*>(a.bias) + n0(q), int(min(int64_t(V), a.n - n0(q))));
#pragma unroll
      for (int e = 0; e < V; ++e) b[q * V + e] = float(p.v[e]);
    }
  }
  f32x4 acc_w[2][KT];
#pragma unroll
  for (int j = 0; j < 2; ++j)
#pragma unroll
    for (int k = 0; k < KT; ++k) acc_w[j][k] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};

  constexpr int XALL = B::ROWS * (KP / V), XP = (XALL + B::THREADS - 1) / B::THREADS;  // x packs, per thread
  constexpr bool XEVEN = XALL % B::THREADS == 0;
  // Inside and edge as in the forward.
  const bool near = a.x_ld <= kNear && a.dl_ld <= kNear && a.g_x_ld <= kNear && a.x_ld > 0 && a.dl_ld > 0;
  const int64_t inside = near && a.m > kSpare ? (a.m - kSpare) / B::ROWS : 0;
  constexpr int XSTEP = B::THREADS / (KP / V);  // rows that one pack a thread covers
  const int x_at = tid % (KP / V) * V, x_count = XEVEN || tid < XALL ? int(a.k) - x_at : 0;
  const uint32_t x_off = x_count > 0 ? uint32_t(tid / (KP / V) * a.x_ld + x_at) : 0u,
                 gx_off = uint32_t(r * a.g_x_ld + (Q == 1 ? 8 : 4) * g);
  const bool tail = a.k != KP || a.n != B::NP;  // packs are masked after the loads have been waited for
  const uint32_t x_ld = uint32_t(a.x_ld), dl_ld = uint32_t(a.dl_ld), gx_ld = uint32_t(a.g_x_ld);  // if near
  const PackMask<T> x_mask = first_of_pack<T>(x_count);
  uint32_t dl_off[Q];
  PackMask<T> dz_mask[Q];
#pragma unroll
  for (int q = 0; q < Q; ++q) {
    dl_off[q] = uint32_t((group * B::GROUP_ROWS + r) * a.dl_ld + (n0(q) < a.n ? n0(q) : 0));
    dz_mask[q] = first_of_pack<T>(int(a.n) - n0(q));
  }
  Pack<T> xr[XP], dr[MT][Q];
  auto load_x_inside = [&](int64_t t) {
    const T* p = x + t * B::ROWS * a.x_ld;
#pragma unroll
    for (int u = 0; u < XP; ++u) xr[u] = load_pack(p + (x_off + u * XSTEP * x_ld));
  };
  auto load_dl_inside = [&](int64_t t) {
    const T* p = dl + t * B::ROWS * a.dl_ld;
#pragma unroll
    for (int i = 0; i < MT; ++i)
#pragma unroll
      for (int q = 0; q < Q; ++q) dr[i][q] = load_pack(p + (dl_off[q] + 16 * i * dl_ld));
  };
  auto load_edge = [&](int64_t t) {
#pragma unroll
    for (int u = 0; u < XP; ++u) {
      const int c = u * B::THREADS + tid;
      const int64_t row = t * B::ROWS + c / (KP / V);
      const int at = c % (KP / V) * V;
      xr[u].v = T(0.0f);
      if ((XEVEN || c < XALL) && row < a.m && at < a.k) xr[u] = load_some(x + row * a.x_ld + at, fresh(int(a.k) - at));
    }
#pragma unroll
    for (int i = 0; i < MT; ++i) {
      const int64_t row = t * B::ROWS + group * B::GROUP_ROWS + 16 * i + r;
#pragma unroll
      for (int q = 0; q < Q; ++q) {
        dr[i][q].v = T(0.0f);
        if (row < a.m && n0(q) < a.n) dr[i][q] = load_some(dl + row * a.dl_ld + n0(q), fresh(int(a.n) - n0(q)));
      }
    }
  };
  __syncthreads();  // W is there
  typename Pack<T>::V fw[2][S];
#pragma unroll
  for (int j = 0; j < 2; ++j)
#pragma unroll
    for (int s = 0; s < S; ++s) fw[j][s] = fragment_of_row(lw, B::KPITCH, 32 * slice + paired_row<T>(j, r), s * D, g);

  // One tile, whose rows are in (or on the way to) xr and dr; next: the tile to ask for meanwhile.
  auto work = [&](auto whole_tile, int64_t t, int64_t next) {
    constexpr bool whole = decltype(whole_tile)::value;
#pragma unroll
    for (int u = 0; u < XP; ++u) {
      const int c = u * B::THREADS + tid;
      if (!XEVEN && c >= XALL) continue;
      if (tail) mask_pack(xr[u], x_mask);
      store_paired(lx + c / (KP / V) * B::KPITCH, c % (KP / V) * V, xr[u]);
    }
    lds_barrier();  // x is there; g_x of the last tile has read dz
    if (whole) load_x_inside(next);
    // dz of this wave's rows and outputs
#pragma unroll
    for (int i = 0; i < MT; ++i) {
      const int lrow = group * B::GROUP_ROWS + 16 * i + r;
      f32x4 z[2] = {f32x4{b[0], b[1], b[2], b[3]}, f32x4{b[4], b[5], b[6], b[7]}};
      if (a.act != GART_ACT_NONE) {
#pragma unroll
        for (int s = 0; s < S; ++s) {
          const auto fx = fragment_of_row(lx, B::KPITCH, lrow, s * D, g);
#pragma unroll
          for (int j = 0; j < 2; ++j) z[j] = Mfma<T>::run(fw[j][s], fx, z[j]);
        }
      }
      float d[8];
      with_activation(a.act, [&](auto act) {
#pragma unroll
        for (int q = 0; q < Q; ++q)
#pragma unroll
          for (int e = 0; e < V; ++e)
            d[q * V + e] = activate_grad<decltype(act)::value>(z[Q == 1 ? e / 4 : q][e % 4], float(dr[i][q].v[e]));
      });
      if (!whole && t * B::ROWS + lrow >= a.m) {  // a row that is not there has a slope all the same
#pragma unroll
        for (int e = 0; e < 8; ++e) d[e] = 0.0f;
      }
#pragma unroll
      for (int q = 0; q < Q; ++q) {
        Pack<T> o, low;
#pragma unroll
        for (int e = 0; e < V; ++e) sum_b[q * V + e] += d[q * V + e];
        if constexpr (PARTS) {
          split_dz<T>(d, o, low);
        } else {
#pragma unroll
          for (int e = 0; e < V; ++e) o.v[e] = T(d[q * V + e]);
        }
        // outputs that are not there are masked: their z is a NaN where x is infinite
        if (tail) mask_pack(o, dz_mask[q]);
        *reinterpret_cast<typename Pack<T>::V*>(lz + lrow * B::NPITCH + n0(q)) = o.v;
        if constexpr (PARTS) {
          if (tail) mask_pack(low, dz_mask[q]);
          *reinterpret_cast<typename Pack<T>::V*>(lz_low + lrow * B::NPITCH + n0(q)) = low.v;
        }
      }
    }
    if (whole) load_dl_inside(next);
    lds_barrier();  // dz is there
    if (a.g_w) {
#pragma unroll
      for (int s = 0; s < B::GROUP_ROWS / D; ++s) {
        const int k0 = group * B::GROUP_ROWS + s * D;
        typename Pack<T>::V fz[2], fz_low[2];
#pragma unroll
        for (int j = 0; j < 2; ++j) {
          fz[j] = fragment_of_columns<T>(lz, B::NPITCH, 2 * slice + j, k0, lane);
          if (PARTS) fz_low[j] = fragment_of_columns<T>(lz_low, B::NPITCH, 2 * slice + j, k0, lane);
        }
#pragma unroll
        for (int k = 0; k < KT; ++k) {
          const auto fx = fragment_of_columns<T>(lx, B::KPITCH, k, k0, lane);
#pragma unroll
          for (int j = 0; j < 2; ++j)
            acc_w[j][k] = PARTS ? mfma_dz<T>(fx, fz[j], fz_low[j], acc_w[j][k]) : Mfma<T>::run(fx, fz[j], acc_w[j][k]);
        }
      }
    }
    if (a.g_x) {
      // 32 rows, or 16 where that leaves waves without, times 32 inputs at a time
      constexpr int IT = B::ROWS / 32 * (KP / 32) >= B::WAVES ? 2 : 1;
      for (int u = wave; u < B::ROWS / (16 * IT) * (KP / 32); u += B::WAVES) {
        const int r0 = u / (KP / 32) * 16 * IT, kt = u % (KP / 32) * 2;
        f32x4 acc[IT][2] = {};
#pragma unroll
        for (int n = 0; n < B::NP; n += D) {
          typename Pack<T>::V fz[IT], fz_low[IT];
#pragma unroll
          for (int i = 0; i < IT; ++i) {
            fz[i] = fragment_of_row(lz, B::NPITCH, r0 + 16 * i + r, n, g);
            if (PARTS) fz_low[i] = fragment_of_row(lz_low, B::NPITCH, r0 + 16 * i + r, n, g);
          }
#pragma unroll
          for (int j = 0; j < 2; ++j) {
            const auto fk = fragment_of_columns<T>(lw, B::KPITCH, kt + j, n, lane);
#pragma unroll
            for (int i = 0; i < IT; ++i)
              acc[i][j] = PARTS ? mfma_dz<T>(fk, fz[i], fz_low[i], acc[i][j]) : Mfma<T>::run(fk, fz[i], acc[i][j]);
          }
        }
        // the next tile's loads are waited for before these stores
#pragma unroll
        for (int i = 0; i < XP; ++i) arrive(xr[i]);
#pragma unroll
        for (int i = 0; i < MT; ++i)
#pragma unroll
          for (int q = 0; q < Q; ++q) arrive(dr[i][q]);
#pragma unroll
        for (int i = 0; i < IT; ++i) {
          const int64_t row = t * B::ROWS + r0 + 16 * i + r;
#pragma unroll
          for (int q = 0; q < Q; ++q) {
            const int64_t k = 16 * kt + (Q == 1 ? 8 * g : 16 * q + 4 * g);
            Pack<T> o;
#pragma unroll
            for (int e = 0; e < V; ++e) {
              const float c = acc[i][Q == 1 ? e / 4 : q][e % 4];
              o.v[e] = T(PARTS ? c * (1.0f / kDzUnit<T>) : c);
            }
            if (whole) {
              if (k < a.k)
                store_some(static_cast<T*>(a.g_x) + t * B::ROWS * a.g_x_ld +
                               ((r0 + 16 * i) * gx_ld + 16 * (kt + q) + gx_off),
                           o, fresh(int(a.k - k)));
            } else if (row < a.m && k < a.k)
              store_some(static_cast<T*>(a.g_x) + row * a.g_x_ld + k, o, fresh(int(a.k - k)));
          }
        }
      }
    }
    lds_barrier();  // x may be replaced
  };
  int64_t t = blockIdx.x;
  if (t < inside) {
    load_x_inside(t);
    load_dl_inside(t);
    for (; t < inside; t += gridDim.x) work(std::true_type{}, t, min(t + int64_t(gridDim.x), inside - 1));
  }
  for (; t < tiles; t += gridDim.x) {
    load_edge(t);
    work(std::false_type{}, t, 0);
  }

  if constexpr (PARTS) {
#pragma unroll
    for (int j = 0; j < 2; ++j)
#pragma unroll
      for (int k = 0; k < KT; ++k) acc_w[j][k] *= 1.0f / kDzUnit<T>;
  }
  // sums of the tile's columns, then those of the row groups, in order
#pragma unroll
  for (int e = 0; e < 8; ++e)
#pragma unroll
    for (int off = 1; off < 16; off <<= 1) sum_b[e] += __shfl_xor(sum_b[e], off);
  if constexpr (B::RG > 1) {
    f32x4* sw = reinterpret_cast<f32x4*>(lds);  // [slice][j][kt][lane]; the loop's last barrier has passed
    float* sb = reinterpret_cast<float*>(lds) + B::NP * KP;
    static_assert((B::NP * KP + B::NP) * 4 <= B::BYTES, "sums fit");
#pragma unroll
    for (int h = 0; h < B::RG; ++h) {
      if (group == h) {
#pragma unroll
        for (int j = 0; j < 2; ++j)
#pragma unroll
          for (int kt = 0; kt < KT; ++kt) {
            f32x4* q = sw + ((slice * 2 + j) * KT + kt) * 64 + lane;
            if (h > 0) acc_w[j][kt] += *q;
            if (h < B::RG - 1) *q = acc_w[j][kt];
          }
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          float* q = sb + n0(e / V) + e % V;
          if (h > 0) sum_b[e] += *q;
          if (h < B::RG - 1 && r == 0) *q = sum_b[e];
        }
      }
      __syncthreads();
    }
    if (group != B::RG - 1) return;
  }
  // One block: the results.  More: this block's part, weights, then bias.
  const bool alone = gridDim.x == 1;
  float* part = partial + int64_t(blockIdx.x) * a.n * (a.k + 1);
  if (a.g_w) {
#pragma unroll
    for (int j = 0; j < 2; ++j) {
      const int64_t n = 32 * slice + 16 * j + r;
      if (n >= a.n) continue;
#pragma unroll
      for (int kt = 0; kt < KT; ++kt) {
        const int64_t k = paired_row<T>(kt, 4 * g);
        const int count = int(min(int64_t(4), a.k - k));
        Pack<float> p;
        p.v = acc_w[j][kt];
        if (!alone && count > 0) store_some(part + n * a.k + k, p, count);
        if (alone) {
#pragma unroll
          for (int e = 0; e < 4; ++e)
            if (e < count) static_cast<T*>(a.g_w)[n * a.g_w_ld + k + e] = T(p.v[e]);
        }
      }
    }
  }
  if (a.g_bias && r == 0) {
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      const int n = n0(e / V) + e % V;
      if (n >= a.n) continue;
      if (alone)
        static_cast<T*>(a.g_bias)[n] = T(sum_b[e]);
      else
        part[a.n * a.k + n] = sum_b[e];
    }
  }
}

// ---- launches --------------------------------------------------------------------
template <typename T, int KP>
hipError_t forward_kp(const LinearArgs& a, hipStream_t s) {
  const int64_t blocks = even_blocks(ceil_div64(ceil_div64(a.m, 32), kForwardWaves), kForwardBlocks);
  const size_t lds = forward_lds(KP, a.n, sizeof(T));
  if (a.k == KP)
    stream_forward_kernel<T, KP, false><<<uint32_t(blocks), 64 * kForwardWaves, lds, s>>>(a);
  else
    stream_forward_kernel<T, KP, true><<<uint32_t(blocks), 64 * kForwardWaves, lds, s>>>(a);
  return hipGetLastError();
}

template <typename T, int KP, int NS>
hipError_t backward_run(const LinearArgs& a, float* partial, hipStream_t s) {
  using B = BackwardShape<T, KP, NS, false>;
  if constexpr (B::FITS) {
    const int64_t tiles = ceil_div64(a.m, B::ROWS);
    const uint32_t blocks = uint32_t(backward_blocks(tiles));
    if constexpr (sizeof(T) == 2) {
      if (dz_in_parts(a.act, sizeof(T))) {
        stream_backward_kernel<T, KP, NS, true><<<blocks, B::THREADS, 0, s>>>(a, partial, tiles);
        return hipGetLastError();
      }
    }
    stream_backward_kernel<T, KP, NS, false><<<blocks, B::THREADS, 0, s>>>(a, partial, tiles);
    return hipGetLastError();
  }
  return hipErrorInvalidValue;
}

template <typename T, int KP>
hipError_t backward_kp(const LinearArgs& a, int ns, float* partial, hipStream_t s) {
  switch (ns) {
    case 1: return backward_run<T, KP, 1>(a, partial, s);
    case 2: return backward_run<T, KP, 2>(a, partial, s);
    case 4: return backward_run<T, KP, 4>(a, partial, s);
    default: return backward_run<T, KP, 8>(a, partial, s);
  }
}

}  // namespace

template <typename T>
hipError_t stream_forward(const LinearArgs& a, hipStream_t s) {
  switch (round_inputs(a.k)) {
    case 32: return forward_kp<T, 32>(a, s);
    case 64: return forward_kp<T, 64>(a, s);
    case 128: return forward_kp<T, 128>(a, s);
    default:
      if constexpr (sizeof(T) == 2) return forward_kp<T, 256>(a, s);
      return hipErrorInvalidValue;
  }
}

template <typename T>
hipError_t stream_backward(const LinearArgs& a, float* partial, hipStream_t s) {
  const BackwardChoice c = choose_backward(a.k, a.n, sizeof(T));
  switch (c.kp) {
    case 32: return backward_kp<T, 32>(a, c.ns, partial, s);
    case 64: return backward_kp<T, 64>(a, c.ns, partial, s);
    case 128: return backward_kp<T, 128>(a, c.ns, partial, s);
    case 256: return backward_kp<T, 256>(a, c.ns, partial, s);
  }
  return hipErrorInvalidValue;
}

}  // namespace gart
