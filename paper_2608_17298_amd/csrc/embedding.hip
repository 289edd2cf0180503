// Embedding lookup with scaling, and its gradient by sorted ids.
//
// Lookup: one thread copies 16 bytes of a row, scaled in float and rounded
// once.  Bound by the bytes of the output.
//
// Gradient: g[v] = scale * sum of the rows whose id is v.  The ids are sorted
// (stable, with their positions), so equal ids stand side by side and a row's
// sum needs no atomics: the order of its terms is their position, whatever the
// schedule.  The sorted positions are cut into units of kUnit, which balances
// the work whatever the ids' distribution; a run of equal ids inside one unit
// is summed and written there, a run that crosses units leaves one partial sum
// a unit and is joined afterwards, in order.
#include <algorithm>

#include "blocks.h"
#include "ops.h"

namespace gart {
namespace {

constexpr int kThreads = 256;
constexpr int kRowsPerThread = 4;
constexpr int kUnit = 128;  // sorted positions per unit

// ---- lookup ------------------------------------------------------------------
// packs: 16-byte packs per row; lanes: threads per row (packs, at most 256);
// rpb: rows a block holds at a time.
template <typename T, typename Id>
__global__ __launch_bounds__(kThreads) void lookup_kernel(const EmbeddingArgs a, int packs, int lanes, int rpb) {
  const T* __restrict__ table = static_cast<const T*>(a.table);
  const Id* __restrict__ ids = static_cast<const Id*>(a.ids);
  T* __restrict__ out = static_cast<T*>(a.out);
  constexpr int V = Pack<T>::N;
  const int sub = threadIdx.x / lanes, lane = threadIdx.x - sub * lanes;
  if (sub >= rpb) return;
  for (int64_t r0 = int64_t(blockIdx.x) * rpb * kRowsPerThread + sub; r0 < a.n;
       r0 += int64_t(gridDim.x) * rpb * kRowsPerThread) {
    int64_t id[kRowsPerThread];
#pragma unroll
    for (int u = 0; u < kRowsPerThread; ++u) {
      const int64_t r = r0 + int64_t(u) * rpb;
      id[u] = r < a.n ? int64_t(ids[r]) : -1;
      if (id[u] >= a.vocab) id[u] = -1;
    }
    for (int p = lane; p < packs; p += lanes) {
      const int64_t c = int64_t(p) * V;
      const int count = int(min(int64_t(V), a.dim - c));
      Pack<T> v[kRowsPerThread];
#pragma unroll
      for (int u = 0; u < kRowsPerThread; ++u) {
        v[u].v = T(0.0f);
        if (id[u] >= 0) v[u] = load_some(table + id[u] * a.table_ld + c, count);
      }
#pragma unroll
      for (int u = 0; u < kRowsPerThread; ++u) {
        const int64_t r = r0 + int64_t(u) * rpb;
#pragma unroll
        for (int e = 0; e < V; ++e) v[u].v[e] = id[u] >= 0 ? T(float(v[u].v[e]) * a.scale) : T(0.0f);
        if (r < a.n) store_some(out + r * a.out_ld + c, v[u], count);
      }
    }
  }
}

// ---- gradient ----------------------------------------------------------------
// Keys of the sort: the id, or vocab (sorted last) where it names no row.
template <typename Id>
__global__ __launch_bounds__(kThreads) void keys_kernel(const Id* __restrict__ ids, int64_t n, int64_t vocab,
                                                        uint32_t* __restrict__ keys, uint32_t* __restrict__ pos) {
  const int64_t i = int64_t(blockIdx.x) * kThreads + threadIdx.x;
  if (i >= n) return;
  const int64_t id = int64_t(ids[i]);
  keys[i] = uint32_t(id >= 0 && id < vocab ? id : vocab);
  pos[i] = uint32_t(i);
}

template <typename T>
__global__ __launch_bounds__(kThreads) void zero_rows_kernel(T* __restrict__ out, int64_t ld, int64_t rows,
                                                             int64_t cols) {
  constexpr int V = Pack<T>::N;
  const int64_t packs = (cols + V - 1) / V, total = rows * packs;
  Pack<T> z;
  z.v = T(0.0f);
  for (int64_t i = int64_t(blockIdx.x) * kThreads + threadIdx.x; i < total; i += int64_t(gridDim.x) * kThreads) {
    const int64_t r = i / packs, c = (i - r * packs) * V;
    store_some(out + r * ld + c, z, int(min(int64_t(V), cols - c)));
  }
}

// Partial sums: partial[2 u] is the part in unit u of a run that began before
// u, partial[2 u + 1] the part in u of a run that begins in u and goes on.
template <typename T>
__global__ __launch_bounds__(kThreads) void unit_sums_kernel(const EmbeddingArgs a, const uint32_t* __restrict__ keys,
                                                             const uint32_t* __restrict__ pos,
                                                             float* __restrict__ partial, int packs, int lanes,
                                                             int upb) {
  const T* __restrict__ rows = static_cast<const T*>(a.rows);
  T* __restrict__ out = static_cast<T*>(a.out);
  constexpr int V = Pack<T>::N;
  const int sub = threadIdx.x / lanes, lane = threadIdx.x - sub * lanes;
  if (sub >= upb) return;
  const int64_t unit = int64_t(blockIdx.x) * upb + sub;
  const int64_t p0 = unit * kUnit, p1 = min(a.n, p0 + kUnit);
  if (p0 >= a.n) return;
  const uint32_t none = uint32_t(a.vocab);
  const uint32_t before = p0 > 0 ? keys[p0 - 1] : none;
  const uint32_t after = p1 < a.n ? keys[p1] : none;
  for (int p = lane; p < packs; p += lanes) {
    const int64_t c = int64_t(p) * V;
    const int count = int(min(int64_t(V), a.dim - c));
    float acc[V] = {};
    uint32_t cur = keys[p0];
    bool first = true;
    auto flush = [&](bool last) {
      if (cur == none) return;
      const bool begun = first && cur == before, goes_on = last && cur == after;
      if (begun || goes_on) {
        float* q = partial + (2 * unit + (begun ? 0 : 1)) * a.dim + c;
        for (int e = 0; e < count; ++e) q[e] = acc[e];
      } else {
        Pack<T> v;
#pragma unroll
        for (int e = 0; e < V; ++e) v.v[e] = T(acc[e] * a.scale);
        store_some(out + int64_t(cur) * a.out_ld + c, v, count);
      }
    };
    for (int64_t i = p0; i < p1; ++i) {
      const uint32_t k = keys[i];
      if (k != cur) {
        flush(false);
        first = false;
        cur = k;
#pragma unroll
        for (int e = 0; e < V; ++e) acc[e] = 0.0f;
      }
      if (k == none) break;
      const Pack<T> v = load_some(rows + int64_t(pos[i]) * a.rows_ld + c, count);
#pragma unroll
      for (int e = 0; e < V; ++e) acc[e] += float(v.v[e]);
    }
    flush(true);
  }
}

// One block per unit whose last run begins there and goes on: adds up the
// run's partial sums.
template <typename T>
__global__ __launch_bounds__(kThreads) void join_kernel(const EmbeddingArgs a, const uint32_t* __restrict__ keys,
                                                        const float* __restrict__ partial) {
  T* __restrict__ out = static_cast<T*>(a.out);
  const int64_t unit = blockIdx.x, p0 = unit * kUnit, p1 = p0 + kUnit;
  if (p1 >= a.n) return;
  const uint32_t cur = keys[p1 - 1];
  if (cur != keys[p1] || cur == uint32_t(a.vocab)) return;      // nothing goes on
  if (p0 > 0 && keys[p0] == cur && keys[p0 - 1] == cur) return;  // began before
  for (int64_t c = threadIdx.x; c < a.dim; c += kThreads) {
    float acc = partial[(2 * unit + 1) * a.dim + c];
    for (int64_t u = unit + 1; u * kUnit < a.n && keys[u * kUnit] == cur; ++u) acc += partial[2 * u * a.dim + c];
    out[int64_t(cur) * a.out_ld + c] = T(acc * a.scale);
  }
}

int bits_for(int64_t v) {  // bits of the largest key v
  int b = 1;
  while ((int64_t(1) << b) <= v) ++b;
  return b;
}

struct GradLayout {
  size_t keys, pos, keys_alt, pos_alt, radix, partial, total;
};

GradLayout grad_layout(int64_t n, int64_t dim) {
  GradLayout L{};
  size_t off = 0;
  auto take = [&](size_t bytes) {
    const size_t o = off;
    off += (bytes + 255) & ~size_t(255);
    return o;
  };
  L.keys = take(size_t(n) * 4);
  L.pos = take(size_t(n) * 4);
  L.keys_alt = take(size_t(n) * 4);
  L.pos_alt = take(size_t(n) * 4);
  L.radix = take(radix_tmp_bytes(n));
  L.partial = take(size_t(ceil_div64(n, kUnit)) * 2 * size_t(dim) * 4);
  L.total = off;
  return L;
}

template <typename T>
hipError_t lookup(const EmbeddingArgs& a, hipStream_t s) {
  if (a.n <= 0 || a.dim <= 0) return hipSuccess;
  const int packs = int(ceil_div64(a.dim, Pack<T>::N)), lanes = std::min(packs, kThreads), rpb = kThreads / lanes;
  const int64_t blocks = std::min<int64_t>(ceil_div64(a.n, int64_t(rpb) * kRowsPerThread), 1 << 20);
  if (a.ids64)
    lookup_kernel<T, int64_t><<<uint32_t(blocks), kThreads, 0, s>>>(a, packs, lanes, rpb);
  else
    lookup_kernel<T, int32_t><<<uint32_t(blocks), kThreads, 0, s>>>(a, packs, lanes, rpb);
  return hipGetLastError();
}

template <typename T>
hipError_t gradient(const EmbeddingArgs& a, hipStream_t s) {
  if (a.vocab <= 0 || a.dim <= 0) return hipSuccess;
  const int packs = int(ceil_div64(a.dim, Pack<T>::N)), lanes = std::min(packs, kThreads), upb = kThreads / lanes;
  const int64_t zero_blocks = std::min<int64_t>(ceil_div64(a.vocab * packs, kThreads), 1 << 16);
  zero_rows_kernel<T><<<uint32_t(zero_blocks), kThreads, 0, s>>>(static_cast<T*>(a.out), a.out_ld, a.vocab, a.dim);
  hipError_t e = hipGetLastError();
  if (e != hipSuccess || a.n <= 0) return e;
  const GradLayout L = grad_layout(a.n, a.dim);
  char* base = static_cast<char*>(a.scratch);
  auto words = [&](size_t off) { return reinterpret_cast<uint32_t*>(base + off); };
  uint32_t *keys = words(L.keys), *pos = words(L.pos);
  const uint32_t blocks = uint32_t(ceil_div64(a.n, kThreads));
  if (a.ids64)
    keys_kernel<int64_t><<<blocks, kThreads, 0, s>>>(static_cast<const int64_t*>(a.ids), a.n, a.vocab, keys, pos);
  else
    keys_kernel<int32_t><<<blocks, kThreads, 0, s>>>(static_cast<const int32_t*>(a.ids), a.n, a.vocab, keys, pos);
  if ((e = hipGetLastError()) != hipSuccess) return e;
  e = radix_sort_u32(keys, pos, words(L.keys_alt), words(L.pos_alt), a.n, bits_for(a.vocab), base + L.radix, s);
  if (e != hipSuccess) return e;
  float* partial = reinterpret_cast<float*>(base + L.partial);
  const int64_t units = ceil_div64(a.n, kUnit);
  unit_sums_kernel<T><<<uint32_t(ceil_div64(units, upb)), kThreads, 0, s>>>(a, keys, pos, partial, packs, lanes, upb);
  if ((e = hipGetLastError()) != hipSuccess) return e;
  if (units > 1) join_kernel<T><<<uint32_t(units - 1), kThreads, 0, s>>>(a, keys, partial);
  return hipGetLastError();
}

}  // namespace

size_t embedding_scratch_bytes(int64_t n, int64_t, int64_t dim) { return n > 0 ? grad_layout(n, dim).total : 0; }

hipError_t launch_embedding(const EmbeddingArgs& a, gart_dtype t, hipStream_t s) {
  if (t == GART_DTYPE_F32) return lookup<float>(a, s);
  if (t == GART_DTYPE_BF16) return lookup<bf16>(a, s);
  return lookup<f16>(a, s);
}

hipError_t launch_embedding_backward(const EmbeddingArgs& a, gart_dtype t, hipStream_t s) {
  if (t == GART_DTYPE_F32) return gradient<float>(a, s);
  if (t == GART_DTYPE_BF16) return gradient<bf16>(a, s);
  return gradient<f16>(a, s);
}

}  // namespace gart
