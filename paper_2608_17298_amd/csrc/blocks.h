// Shared by the learned blocks (embedding, linear layer, dropout): element
// types, 16-byte accesses of any alignment, and the launchers' arguments.
#pragma once

#include <hip/hip_runtime.h>

#include <cstddef>
#include <cstdint>

#include "../../include/gart.h"

namespace gart {

using bf16 = __bf16;
using f16 = _Float16;

// 16 bytes at any address: gfx950 takes unaligned global accesses, so odd row
// strides and odd column counts keep the wide form (an access that spans two
// lines costs both).
struct __attribute__((packed)) packed16 {
  uint32_t w[4];
};

template <typename T>
struct Pack {  // the elements of one 16-byte access
  static constexpr int N = 16 / int(sizeof(T));
  typedef T V __attribute__((ext_vector_type(16 / sizeof(T))));
  V v;
};

template <typename T>
__device__ __forceinline__ Pack<T> load_pack(const T* p) {
  const packed16 q = *reinterpret_cast<const packed16*>(p);
  Pack<T> r;
  __builtin_memcpy(&r, &q, 16);
  return r;
}

template <typename T>
__device__ __forceinline__ void store_pack(T* p, const Pack<T>& r) {
  packed16 q;
  __builtin_memcpy(&q, &r, 16);
  *reinterpret_cast<packed16*>(p) = q;
}

// The same past the caches, for full lines that nothing is going to read soon.
template <typename T>
__device__ __forceinline__ void store_past(T* p, const Pack<T>& r) {
  typedef uint32_t u32x4 __attribute__((ext_vector_type(4), aligned(2)));
  u32x4 q;
  __builtin_memcpy(&q, &r, 16);
  __builtin_nontemporal_store(q, reinterpret_cast<u32x4*>(p));
}

// A value the compiler takes for new, so that comparisons with it are made where
// they are needed and not held through a loop (in scalar registers, which spill).
__device__ __forceinline__ int fresh(int v) {
  asm volatile("" : "+v"(v));
  return v;
}

// Loaded values are waited for here.  Loads and stores retire in order, so a
// wait placed after younger stores would wait for those as well.
template <typename V>
__device__ __forceinline__ void arrive(V& v) {
  typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
  u32x4 w;
  __builtin_memcpy(&w, &v, 16);
  asm volatile("" : "+v"(w));
  __builtin_memcpy(&v, &w, 16);
}

// The first `count` elements at p, the rest zero.
template <typename T>
__device__ __forceinline__ Pack<T> load_some(const T* p, int count) {
  if (count >= Pack<T>::N) return load_pack(p);
  Pack<T> r;
#pragma unroll
  for (int e = 0; e < Pack<T>::N; ++e) r.v[e] = e < count ? p[e] : T(0.0f);
  return r;
}

// Bits of a pack's first `count` elements: for packs that may be read whole in
// any case (there are rows after them), without a branch.
template <typename T>
struct PackMask {
  uint32_t w[4];
};

template <typename T>
__device__ __forceinline__ PackMask<T> first_of_pack(int count) {
  PackMask<T> m;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    if constexpr (sizeof(T) == 4)
      m.w[i] = count > i ? ~0u : 0u;
    else
      m.w[i] = count > 2 * i + 1 ? ~0u : count == 2 * i + 1 ? 0xFFFFu : 0u;
  }
  return m;
}

template <typename T>
__device__ __forceinline__ void mask_pack(Pack<T>& v, const PackMask<T>& m) {
  uint32_t w[4];
  __builtin_memcpy(w, &v, 16);
#pragma unroll
  for (int i = 0; i < 4; ++i) w[i] &= m.w[i];
  __builtin_memcpy(&v, w, 16);
}

template <typename T>
__device__ __forceinline__ void store_some(T* p, const Pack<T>& r, int count) {
  if (count >= Pack<T>::N) {
    store_pack(p, r);
    return;
  }
#pragma unroll
  for (int e = 0; e < Pack<T>::N; ++e)
    if (e < count) p[e] = r.v[e];
}

inline int64_t ceil_div64(int64_t a, int64_t b) { return (a + b - 1) / b; }
inline size_t dtype_bytes(gart_dtype t) { return t == GART_DTYPE_F32 ? 4 : 2; }

// ---- embedding.hip ---------------------------------------------------------
struct EmbeddingArgs {
  const void* ids;  // [n] int32 or int64
  bool ids64;
  int64_t n, vocab, dim;
  float scale;
  const void* table;  // forward: [vocab, dim]
  int64_t table_ld;
  const void* rows;  // backward: dl_dout [n, dim]
  int64_t rows_ld;
  void* out;  // forward: [n, dim]; backward: g_table [vocab, dim]
  int64_t out_ld;
  void* scratch;
};
size_t embedding_scratch_bytes(int64_t n, int64_t vocab, int64_t dim);
// whether the gradient's sums fit the 2^32 threads of a launch
bool embedding_backward_launchable(int64_t n, int64_t dim, gart_dtype t);
hipError_t launch_embedding(const EmbeddingArgs& a, gart_dtype t, hipStream_t s);
hipError_t launch_embedding_backward(const EmbeddingArgs& a, gart_dtype t, hipStream_t s);

// ---- dropout.hip -----------------------------------------------------------
struct DropoutArgs {
  const void *x, *residual;  // residual may be NULL
  void* y;
  int64_t rows, cols, x_ld, residual_ld, y_ld;
  uint32_t threshold;  // an element is dropped where its 16 random bits are below this
  float scale;
  uint64_t seed, offset;
};
hipError_t launch_dropout(const DropoutArgs& a, gart_dtype t, hipStream_t s);

// ---- linear.hip ------------------------------------------------------------
struct LinearArgs {
  int64_t m, k, n;  // rows, inputs, outputs
  gart_activation act;
  const void *x, *w, *bias, *residual, *dl;
  int64_t x_ld, w_ld, residual_ld, dl_ld;
  void *y, *g_x, *g_w, *g_bias;
  int64_t y_ld, g_x_ld, g_w_ld;
  void* scratch;
};
// -1 if the sizes are beyond what a launch can index
int64_t linear_scratch_bytes(int64_t m, int64_t k, int64_t n, gart_dtype t);
int64_t linear_backward_scratch_bytes(int64_t m, int64_t k, int64_t n, gart_dtype t, gart_activation act);
hipError_t launch_linear(const LinearArgs& a, gart_dtype t, hipStream_t s);
hipError_t launch_linear_backward(const LinearArgs& a, gart_dtype t, hipStream_t s);

}  // namespace gart
