// Device code shared by the linear layer's kernels: matrix instructions,
// activations, fragments in LDS; and the launchers' sub-plans.
#pragma once

#include <type_traits>

#include "blocks.h"
#include "linear_cut.h"

namespace gart {

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
// logistic function g(u) = 1 / (1 + exp(-u)) = 1 / (1 + 2^(-u log2 e)).  The
// exponent is one rounded product: it is off by the size of z's own rounding.
// z is held where g is exactly 0 or 1 in float, so that an infinite z meets no
// infinity times 0; these minima and maxima let a NaN through.
constexpr float kGelu = 1.5957691216057308f;  // 2 sqrt(2 / pi)
constexpr float kCubic = 0.044715f;
constexpr float kLog2e = 1.4426950408889634f;

template <gart_activation ACT>
constexpr float kEdge = ACT == GART_ACT_GELU ? 12.0f : 104.0f;

// exp(-u)
template <gart_activation ACT>
__device__ __forceinline__ float gate_exp(float z) {
  float h;
  if constexpr (ACT == GART_ACT_GELU)
    h = z * fmaf(z * z, -kGelu * kCubic * kLog2e, -kGelu * kLog2e);
  else
    h = z * -kLog2e;
  return __builtin_amdgcn_exp2f(h);
}

template <gart_activation ACT>
__device__ __forceinline__ float activate(float z) {
  if constexpr (ACT == GART_ACT_NONE) return z;
  if constexpr (ACT == GART_ACT_RELU) return z < 0.0f ? 0.0f : z;  // a NaN stays
  const float c = __builtin_elementwise_maximum(z, -kEdge<ACT>);
  return c * __builtin_amdgcn_rcpf(1.0f + gate_exp<ACT>(c));
}

// dl times act'(z) = g + z u' g (1 - g), where 1 - g is exp(-u) g: the difference
// would lose what the factor z u' brings back (gelu's slope near z = 4: 2e-6 off).
template <gart_activation ACT>
__device__ __forceinline__ float activate_grad(float z, float dl) {
  if constexpr (ACT == GART_ACT_NONE) return dl;
  if constexpr (ACT == GART_ACT_RELU) return z <= 0.0f ? 0.0f : dl;
  const float c = __builtin_elementwise_minimum(__builtin_elementwise_maximum(z, -kEdge<ACT>), kEdge<ACT>);
  const float x = gate_exp<ACT>(c), g = __builtin_amdgcn_rcpf(1.0f + x);
  const float s = ACT == GART_ACT_GELU ? c * fmaf(3.0f * kCubic * kGelu * c, c, kGelu) : c;
  return dl * fmaf(s * g, fminf(x, 0x1p126f) * g, g);  // an infinite exp(-u) has g = 0
}

// f(integral constant of act): one branch a block of elements, none between them
template <typename F>
__device__ __forceinline__ void with_activation(gart_activation act, F&& f) {
  switch (act) {
    case GART_ACT_NONE: f(std::integral_constant<gart_activation, GART_ACT_NONE>{}); break;
    case GART_ACT_RELU: f(std::integral_constant<gart_activation, GART_ACT_RELU>{}); break;
    case GART_ACT_SILU: f(std::integral_constant<gart_activation, GART_ACT_SILU>{}); break;
    case GART_ACT_GELU: f(std::integral_constant<gart_activation, GART_ACT_GELU>{}); break;
  }
}

// ---- dz in two parts -----------------------------------------------------------
// 16 bits: dz = dl act'(z), the operand of two products, is more exact than its
// inputs, so it enters them as the sum of two numbers of the type, high + low,
// with one matrix instruction each: off by 2^-15 (bf16) or 2^-20 (f16) of itself.
// Where act' is 0 or 1 (none, relu) dz is of the type anyway.
//
// The high part is dz, less one unit of its last place as a float, cut off to the
// type.  So both parts have dz's sign and neither is 0 unless dz is (or is as small
// as the type's smallest number): an infinite operand gives dz's infinity, not
// the NaN of infinity times 0 or of two signs; and an infinite dz leaves a finite
// high and an infinite low part.  float16 holds dz times kDzUnit, as |act'| passes
// 1, and the low part times kDzLow, as small ones would be lost below 2^-24.
template <typename T>
constexpr float kDzUnit = std::is_same<T, f16>::value ? 0.5f : 1.0f;
template <typename T>
constexpr float kDzLow = std::is_same<T, f16>::value ? 1024.0f : 1.0f;

inline bool dz_in_parts(gart_activation act, size_t es) {
  return es == 2 && (act == GART_ACT_SILU || act == GART_ACT_GELU);
}

// Two elements: their high parts, the first one's in the low bits, and their low parts.
template <typename T>
__device__ __forceinline__ void split_dz(float d0, float d1, uint32_t& high, uint32_t& low) {
  // 0 is added after the product, which may underflow to -0: neither zero has a number below it
  const float h[2] = {d0 * kDzUnit<T> + 0.0f, d1 * kDzUnit<T> + 0.0f};
  uint32_t u[2];
#pragma unroll
  for (int e = 0; e < 2; ++e) u[e] = __builtin_elementwise_sub_sat(__builtin_bit_cast(uint32_t, h[e]), 1u);
  if constexpr (std::is_same<T, bf16>::value) {
    high = __builtin_amdgcn_perm(u[1], u[0], 0x07060302u);
    bf16 l[2];
#pragma unroll
    for (int e = 0; e < 2; ++e) l[e] = bf16(h[e] - __builtin_bit_cast(float, u[e] & 0xFFFF0000u));
    __builtin_memcpy(&low, l, 4);
  } else {
    const auto t = __builtin_amdgcn_cvt_pkrtz(__builtin_bit_cast(float, u[0]), __builtin_bit_cast(float, u[1]));
    const auto l = __builtin_amdgcn_cvt_pkrtz((h[0] - float(t[0])) * kDzLow<T>, (h[1] - float(t[1])) * kDzLow<T>);
    __builtin_memcpy(&high, &t, 4);
    __builtin_memcpy(&low, &l, 4);
  }
}

template <typename T>
__device__ __forceinline__ void split_dz(float d, T& high, T& low) {
  uint32_t h, l;
  split_dz<T>(d, 0.0f, h, l);
  __builtin_memcpy(&high, &h, 2);
  __builtin_memcpy(&low, &l, 2);
}

template <typename T>
__device__ __forceinline__ void split_dz(const float* d, Pack<T>& high, Pack<T>& low) {
  uint32_t h[4], l[4];
#pragma unroll
  for (int e = 0; e < 4; ++e) split_dz<T>(d[2 * e], d[2 * e + 1], h[e], l[e]);
  __builtin_memcpy(&high, h, 16);
  __builtin_memcpy(&low, l, 16);
}

// c + kDzUnit a dz
template <typename T>
__device__ __forceinline__ f32x4 mfma_dz(typename Pack<T>::V a, typename Pack<T>::V high, typename Pack<T>::V low,
                                         f32x4 c) {
  if constexpr (kDzLow<T> == 1.0f) {
    return Mfma<T>::run(a, high, Mfma<T>::run(a, low, c));
  } else {
    const f32x4 t = Mfma<T>::run(a, low, f32x4{0.0f, 0.0f, 0.0f, 0.0f});
    c = Mfma<T>::run(a, high, c);
#pragma unroll
    for (int e = 0; e < 4; ++e) c[e] = fmaf(t[e], 1.0f / kDzLow<T>, c[e]);
    return c;
  }
}

// ---- fragments ---------------------------------------------------------------
// A 16-bit fragment holds eight consecutive k of a row, lanes r = lane % 16
// over the rows and g = lane / 16 over the k (8 g ..); a float one four (4 g ..).
template <typename T>
constexpr int kDepth = sizeof(T) == 2 ? 32 : 16;  // k per fragment

// Rows of a fragment of the products' first operand, which become a lane's
// output columns.  16 bits: tiles 2q and 2q+1 together hold 32 columns, eight
// consecutive ones a lane.  float: a lane's four are 16 bytes already.
template <typename T>
__device__ __forceinline__ int paired_row(int tile, int r) {
  return sizeof(T) == 2 ? 32 * (tile / 2) + 8 * (r / 4) + 4 * (tile % 2) + r % 4 : 16 * tile + r;
}

// From LDS rows along k.
template <typename T>
__device__ __forceinline__ typename Pack<T>::V fragment_of_row(const T* lds, int pitch, int row, int k0, int g) {
  return *reinterpret_cast<const typename Pack<T>::V*>(lds + row * pitch + k0 + Pack<T>::N * g);
}

// A pack of a row (columns at ..) into LDS so that the rows a paired tile takes
// stand side by side: of 16 bits, the first halves of a block of 32 columns come
// before the second halves.  fragment_of_columns, unpaired, of such rows yields
// the paired columns without bank conflicts (paired from plain rows: two-way);
// along rows, two operands stored alike still agree on k.
template <typename T>
__device__ __forceinline__ void store_paired(T* row, int at, const Pack<T>& p) {
  if constexpr (sizeof(T) == 4) {
    *reinterpret_cast<typename Pack<T>::V*>(row + at) = p.v;
  } else {
    uint2 h[2];
    __builtin_memcpy(h, &p, 16);
    T* q = row + at / 32 * 32 + at % 32 / 2;
    *reinterpret_cast<uint2*>(q) = h[0];
    *reinterpret_cast<uint2*>(q + 16) = h[1];
  }
}

// 16 bits, from lines across k: the lanes of a group of 16 name four lines times
// 16 columns, four columns a lane, and the transposing load gives each lane the
// four k of its column; the other four k lie `down` elements on.
template <typename T>
__device__ __forceinline__ typename Pack<T>::V transposed_pair(const T* lds, int down) {
  typedef short s16x4 __attribute__((ext_vector_type(4)));
  typedef __attribute__((address_space(3))) s16x4* lds_ptr;
  const s16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_ptr)(lds));
  const s16x4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_ptr)(lds + down));
  typename Pack<T>::V v;
  __builtin_memcpy(&v, &lo, 8);
  __builtin_memcpy(reinterpret_cast<char*>(&v) + 8, &hi, 8);
  return v;
}

// From LDS lines across k (line k holds the rows' elements side by side).
template <typename T>
__device__ __forceinline__ typename Pack<T>::V fragment_of_columns(const T* lds, int pitch, int tile, int k0,
                                                                   int lane) {
  const int r = lane % 16, g = lane / 16;
  typename Pack<T>::V v;
  if constexpr (sizeof(T) == 4) {
    const T* q = lds + (k0 + 4 * g) * pitch + 16 * tile + r;
#pragma unroll
    for (int t = 0; t < 4; ++t) v[t] = q[t * pitch];
  } else {
    v = transposed_pair(lds + (k0 + 8 * g + r / 4) * pitch + 16 * tile + 4 * (r % 4), 4 * pitch);
  }
  return v;
}

// A barrier that orders the block's LDS accesses alone: loads and stores of
// global memory stay in flight across it (__syncthreads waits for them all).
__device__ __forceinline__ void lds_barrier() {
  __builtin_amdgcn_fence(__ATOMIC_RELEASE, "workgroup", "local");
  __builtin_amdgcn_s_barrier();
  __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "workgroup", "local");
}

// ---- how the work is cut (linear_cut.h, linear.hip) -----------------------------------
constexpr int kJoinRows = 32;          // rows per column sum of a joined dz
constexpr int kSumRows = 256;          // rows per column sum of dl
// Rows up to which every block takes all of them, and inputs, of 16 and of 32 bits,
// up to which it does with so many rows (linear_rows.h).
constexpr int64_t kFewRows = 32, kFewRowsShort = 4096, kFewRowsFloat = 2048;
constexpr int64_t kMoreRows = 64, kMoreRowsShort = 2048, kMoreRowsFloat = 512;

// 16-bit gradients with few elements of dz, and inputs, take two launches of
// their own (linear_small.h), unless one block streams the rows past a small weight.
constexpr int64_t kSmallElements = 1024;
constexpr int64_t kSmallInputs = 16384;
constexpr int64_t kSmallStreamInputs = 128, kSmallStreamWeight = 8192;

struct BackwardPlan {
  bool small, stream;
  int64_t parts;  // partial sums (stream)
  int64_t dz_ld, dz_low;  // dz_low: elements from dz's high parts to the low ones, or 0
  size_t dz, partial, sums, total;
};
BackwardPlan backward_plan(int64_t m, int64_t k, int64_t n, gart_dtype t, gart_activation act);

template <typename T>
constexpr gart_dtype kType = sizeof(T) == 4                  ? GART_DTYPE_F32
                             : std::is_same<T, bf16>::value ? GART_DTYPE_BF16
                                                            : GART_DTYPE_F16;

// ---- linear_rows.h, linear_stream.h, linear_gemm.h: one of each per type -----------
inline bool few_rows(int64_t m, int64_t k, int64_t n, size_t es) {
  return n <= int64_t(1) << 24 && ((m <= kFewRows && k <= (es == 2 ? kFewRowsShort : kFewRowsFloat)) ||
                                   (m <= kMoreRows && k <= (es == 2 ? kMoreRowsShort : kMoreRowsFloat)));
}
// y, or dz and g_bias (may be NULL), of few rows; dz_low: elements from
// dz's high parts to the low ones, 0 if it is not in parts
template <typename T>
hipError_t rows_forward(const LinearArgs& a, hipStream_t s);
template <typename T>
hipError_t rows_dz(const LinearArgs& a, void* dz, int64_t dz_ld, int64_t dz_low, hipStream_t s);

// Layers whose weight fits LDS: the rows stream past it once.
bool stream_forward_fits(int64_t k, int64_t n, size_t es);
// Parts whose partial sums the backward leaves in partial [parts, n k + n] if
// they are more than one (0: the layer does not fit).
int64_t stream_backward_parts(int64_t m, int64_t k, int64_t n, size_t es);
template <typename T>
hipError_t stream_forward(const LinearArgs& a, hipStream_t s);
template <typename T>
hipError_t stream_backward(const LinearArgs& a, float* partial, hipStream_t s);

template <typename T>
hipError_t gemm_forward(const LinearArgs& a, hipStream_t s);
// everything after the plan, streams included
template <typename T>
hipError_t gemm_backward(const LinearArgs& a, hipStream_t s);

}  // namespace gart
