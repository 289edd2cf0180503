// Embedding lookup with scaling, and its gradient by sorted ids.
//
// Lookup: one thread copies 16 bytes of two rows, scaled in float and rounded
// once.  Bound by the bytes of the output: 1M rows of 48 f32 take 38 us, 5.5 TB/s.
//
// Gradient: g[v] = scale * sum of the rows whose id is v.  The ids are sorted
// (stable, with their positions), so equal ids stand side by side and a row's
// sum needs no atomics: the order of its terms is their position, whatever the
// schedule.  The sorted positions are cut into units of equal length, which balances
// the work whatever the ids' distribution; a run of equal ids is summed in its
// units, joined in the block's LDS and, where it crosses blocks, afterwards
// from their partial sums, always in order.
//
// 1M rows of 64 bf16 into 4096 take 84 us: the sort's two passes 42 with the
// clearing, the sums 28 to 30 (rows of 128 bytes at random, 4.5 TB/s), the join
// across blocks 7.
#include <algorithm>

#include "blocks.h"
#include "ops.h"
#include "sort_device.h"

namespace gart {
namespace {

typedef float f32x4 __attribute__((ext_vector_type(4)));

constexpr int kThreads = 256;
constexpr int kRowsPerThread = 2;
constexpr int kBatch = 8;            // rows in flight per thread of the gradient
// Bytes of a lookup's output up to which the reader behind it still finds it in
// the caches: lookup and linear layer of 200k rows of 48 f32, 32.0 us written
// through and 33.3 past them; of 1M rows 109 and 96.
constexpr int64_t kCached = 64 << 20;
constexpr int kMinUnit = 8, kMaxUnit = 64;
constexpr int64_t kUnitThreads = 262144;

// First column of a row's pack p.  The last pack of a row ends with the row and
// overlaps the one before, which computes and stores the same values there: so
// odd columns need no accesses of single elements (gradient of 8191 ids, 1023
// f16: the sums 9 us, element by element 12).
template <typename T>
__device__ __forceinline__ int64_t pack_column(int64_t p, int64_t cols) {
  return max(int64_t(0), min(p * Pack<T>::N, cols - Pack<T>::N));
}

// ---- lookup ------------------------------------------------------------------
// packs: 16-byte packs per row; lanes: threads per row (packs, at most 256);
// rpb: rows a block holds at a time.
template <typename T, typename Id, bool PAST>
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
      const int64_t c = pack_column<T>(p, a.dim);
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
        if (r >= a.n) continue;
        if (PAST && count >= V)
          store_past(out + r * a.out_ld + c, v[u]);
        else
          store_some(out + r * a.out_ld + c, v[u], count);
      }
    }
  }
}

// ---- gradient ----------------------------------------------------------------
template <typename T>
__device__ __forceinline__ void zero_rows(T* __restrict__ out, int64_t ld, int64_t rows, int64_t cols, int64_t first,
                                          int64_t step) {
  constexpr int V = Pack<T>::N;
  const int64_t packs = (cols + V - 1) / V;
  Pack<T> z;
  z.v = T(0.0f);
  if (ld == cols) {  // one run of elements
    const int64_t total = rows * cols;
    for (int64_t i = first * V; i < total; i += step * V) {
      if (total - i >= V)
        store_past(out + i, z);  // 8191 ids into 50021 rows of 1023 f16: 42 us, through the caches 58
      else
        store_some(out + i, z, int(total - i));
    }
    return;
  }
  for (int64_t i = first; i < rows * packs; i += step) {
    const int64_t r = i / packs, c = pack_column<T>(i - r * packs, cols);
    store_some(out + r * ld + c, z, int(min(int64_t(V), cols - c)));
  }
}

// The first `counting` blocks count the ids' first digits, the others clear the
// table's gradient (with no ids, all of them do).
template <typename T, typename Id>
__global__ __launch_bounds__(kThreads) void count_and_zero_kernel(const EmbeddingArgs a, uint32_t* __restrict__ counts,
                                                                  int counting, bool by_block) {
  static_assert(kThreads == kSortThreads, "a block counts as one of the sort's");
  if (int(blockIdx.x) < counting) {
    radix_count<kIdItems>(IdSource<Id>{static_cast<const Id*>(a.ids), a.vocab}, a.n, 0, counts, counting, by_block);
    return;
  }
  zero_rows(static_cast<T*>(a.out), a.out_ld, a.vocab, a.dim,
            int64_t(blockIdx.x - counting) * kThreads + threadIdx.x, int64_t(gridDim.x - counting) * kThreads);
}

// Up to kSmallPairs ids: the first block sorts them while the others clear the
// table's gradient (8191 ids into 50021 rows of 1023 f16: 19 us for both).
template <typename T, typename Id>
__global__ __launch_bounds__(kSmallThreads) void sort_and_zero_kernel(const EmbeddingArgs a,
                                                                      uint32_t* __restrict__ keys,
                                                                      uint32_t* __restrict__ pos, int bits) {
  if (blockIdx.x > 0) {
    zero_rows(static_cast<T*>(a.out), a.out_ld, a.vocab, a.dim, int64_t(blockIdx.x - 1) * kSmallThreads + threadIdx.x,
              int64_t(gridDim.x - 1) * kSmallThreads);
    return;
  }
  const IdSource<Id> source{static_cast<const Id*>(a.ids), a.vocab};
  if (a.n <= kSmallThreads)
    radix_small<1>(source, keys, pos, int(a.n), bits);
  else
    radix_small<8>(source, keys, pos, int(a.n), bits);
}

// Sums of a block's units.  A thread owns 16 bytes of the rows of one unit.
// kBatch rows are asked for before any of them is added, whatever their keys
// (one row at a time left the kernel waiting for memory: 141 us at 1M rows of
// 64 bf16).  Runs that cross units meet in LDS, in order; what crosses blocks
// leaves partial sums: partial[2 b] is the part in block b of a run that began
// before b, partial[2 b + 1] the part of a run that begins in b and goes on.
template <typename T>
__global__ __launch_bounds__(kThreads) void unit_sums_kernel(const EmbeddingArgs a, const uint32_t* __restrict__ keys,
                                                             const uint32_t* __restrict__ pos,
                                                             float* __restrict__ partial, int unit_rows, int packs,
                                                             int lanes, int upb) {
  constexpr int V = Pack<T>::N;
  __shared__ __attribute__((aligned(16))) float s_head[kThreads][V];  // of the unit's first run, if it began before
  __shared__ bool s_whole[kThreads];  // the unit is one run that began before and goes on
  const T* __restrict__ rows = static_cast<const T*>(a.rows);
  T* __restrict__ out = static_cast<T*>(a.out);
  const int sub = threadIdx.x / lanes, lane = threadIdx.x - sub * lanes;
  const int64_t block_p0 = int64_t(blockIdx.x) * upb * unit_rows, p0 = block_p0 + int64_t(sub) * unit_rows;
  const int64_t p1 = min(a.n, p0 + unit_rows);
  const int units = int(min(int64_t(upb), (a.n - block_p0 + unit_rows - 1) / unit_rows));
  const bool active = sub < units;
  const uint32_t none = uint32_t(a.vocab);
  const uint32_t before = active && p0 > 0 ? keys[p0 - 1] : none;
  const uint32_t after = active && p1 < a.n ? keys[p1] : none;
  for (int base = 0; base < packs; base += lanes) {
    const int p = base + lane;
    const bool mine = active && p < packs;
    const int64_t c = pack_column<T>(p, a.dim);
    const int count = int(min(int64_t(V), a.dim - c));
    float acc[V] = {};
    uint32_t cur = mine ? keys[p0] : none;
    bool first = true;
    auto put = [&](uint32_t key, const float* sum) {
      Pack<T> v;
#pragma unroll
      for (int e = 0; e < V; ++e) v.v[e] = T(sum[e] * a.scale);
      store_some(out + int64_t(key) * a.out_ld + c, v, count);
    };
    auto put_partial = [&](int which, const float* sum) {
      float* q = partial + (2 * int64_t(blockIdx.x) + which) * a.dim + c;
#pragma unroll
      for (int h = 0; h < V / 4; ++h) {
        Pack<float> f;
#pragma unroll
        for (int e = 0; e < 4; ++e) f.v[e] = sum[4 * h + e];
        if (count > 4 * h) store_some(q + 4 * h, f, count - 4 * h);
      }
    };
    auto keep_head = [&] {
#pragma unroll
      for (int e = 0; e < V; ++e) s_head[threadIdx.x][e] = acc[e];
    };
    if (mine) {
      for (int64_t i = p0; i < p1; i += kBatch) {
        uint32_t k[kBatch], at[kBatch];  // loaded four at a time: 1M rows of 64 bf16 85 us, one at a time 97
        Pack<T> v[kBatch];
        if (i + kBatch <= p1) {
#pragma unroll
          for (int u = 0; u < kBatch; u += 4) {
            const packed16 kq = *reinterpret_cast<const packed16*>(keys + i + u);
            const packed16 aq = *reinterpret_cast<const packed16*>(pos + i + u);
#pragma unroll
            for (int e = 0; e < 4; ++e) {
              k[u + e] = kq.w[e];
              at[u + e] = aq.w[e];
            }
          }
        } else {
#pragma unroll
          for (int u = 0; u < kBatch; ++u) {
            k[u] = i + u < p1 ? keys[i + u] : none;
            at[u] = i + u < p1 ? pos[i + u] : 0u;
          }
        }
#pragma unroll
        for (int u = 0; u < kBatch; ++u) {
          v[u].v = T(0.0f);
          if (k[u] != none) v[u] = load_some(rows + int64_t(at[u]) * a.rows_ld + c, count);
        }
#pragma unroll
        for (int u = 0; u < kBatch; ++u) {
          if (i + u < p1 && k[u] != cur) {  // the run ends inside the unit
            if (first && cur == before)
              keep_head();
            else
              put(cur, acc);
            first = false;
            cur = k[u];
#pragma unroll
            for (int e = 0; e < V; ++e) acc[e] = 0.0f;
          }
#pragma unroll
          for (int e = 0; e < V; ++e) acc[e] += float(v[u].v[e]);
        }
      }
    }
    // the unit's last run: acc, key cur
    const bool there = mine && cur != none, begun = there && first && cur == before, goes_on = there && cur == after;
    if (begun) keep_head();
    if (there && !begun && !goes_on) put(cur, acc);
    if (mine) s_whole[threadIdx.x] = begun && goes_on;
    __syncthreads();
    // adds the units after sub to acc while their first run is the one before's; true if it leaves the block
    auto follow = [&](bool open) {
      for (int u = sub + 1; open && u < units; ++u) {
        const int t = u * lanes + lane;
#pragma unroll
        for (int e = 0; e < V; ++e) acc[e] += s_head[t][e];
        open = s_whole[t];
      }
      return open;
    };
    if (there && !begun && goes_on) {
      if (follow(true))
        put_partial(1, acc);
      else
        put(cur, acc);
    }
    if (mine && sub == 0 && before != none && keys[p0] == before) {  // began before the block
#pragma unroll
      for (int e = 0; e < V; ++e) acc[e] = s_head[threadIdx.x][e];
      follow(s_whole[threadIdx.x]);
      put_partial(0, acc);
    }
    __syncthreads();
  }
}

// Joins the runs that cross the blocks above, its units here: unit u's last run
// begins there and goes on if the key at its end equals the next unit's first,
// and that many further units hold a part of it.  A wave takes one unit; a run that goes on over
// kLongRun further units (at most one begins in a block's 16) is left to the
// block's waves together.  Lanes are spread over a group of columns (four a
// lane; blockIdx.y counts the groups) and, where columns are few, over the
// run's units; the shares are added in a fixed order.
constexpr int kJoinThreads = 1024;
constexpr int kJoinWaves = kJoinThreads / 64;
constexpr int kLongRun = kJoinWaves;
constexpr int kJoinColumns = 256;

// Sum over every step-th of a run's parts, from `first` on: part 0 is the tail
// of `unit`, part u the head of unit + u.
__device__ __forceinline__ f32x4 run_share(const float* __restrict__ partial, int64_t dim, int64_t unit, int64_t more,
                                           int64_t c, int first, int step) {
  f32x4 s = {0.0f, 0.0f, 0.0f, 0.0f};
  const int count = int(min(int64_t(4), dim - c));
#pragma unroll 4
  for (int64_t u = first; u <= more; u += step)
    s += load_some(partial + (u == 0 ? 2 * unit + 1 : 2 * (unit + u)) * dim + c, count).v;
  return s;
}

template <typename T>
__global__ __launch_bounds__(kJoinThreads) void join_kernel(const EmbeddingArgs a, const uint32_t* __restrict__ keys,
                                                            const float* __restrict__ partial, int unit_rows,
                                                            int64_t units) {
  __shared__ int s_long;  // the wave whose unit begins a long run, or -1
  __shared__ f32x4 s_sum[kJoinThreads];
  T* __restrict__ out = static_cast<T*>(a.out);
  const int tid = threadIdx.x, lane = tid % 64, wave = tid / 64;
  const int64_t base = int64_t(blockIdx.x) * kJoinWaves, unit = base + wave;
  const int64_t p0 = unit * unit_rows, p1 = p0 + unit_rows;
  const uint32_t none = uint32_t(a.vocab);
  if (tid == 0) s_long = -1;
  __syncthreads();
  bool mine = unit < units && p1 < a.n;
  uint32_t cur = none;
  if (mine) {
    cur = keys[p1 - 1];
    mine = cur != none && cur == keys[p1] && !(p0 > 0 && keys[p0] == cur && keys[p0 - 1] == cur);
  }
  int more = 0;  // further units with a part of the run
  if (mine) {
    const int64_t q = p1 + int64_t(lane) * unit_rows;
    const uint64_t other = ~__ballot(lane < kLongRun && q < a.n && keys[q] == cur);
    more = __builtin_ctzll(other);
    if (more == kLongRun && lane == 0) s_long = wave;
  }
  auto store = [&](uint32_t key, int64_t c, f32x4 s) {
#pragma unroll
    for (int e = 0; e < 4; ++e)
      if (c + e < a.dim) out[int64_t(key) * a.out_ld + c + e] = T(s[e] * a.scale);
  };
  // columns of this block, and lanes over them: a power of two
  const int64_t c0 = int64_t(blockIdx.y) * kJoinColumns;
  const int quads = int((min(int64_t(kJoinColumns), a.dim - c0) + 3) / 4);
  int w = 1;
  while (w < quads) w *= 2;
  const int64_t c = c0 + int64_t(lane % w) * 4;
  if (more > 0 && more < kLongRun) {
    f32x4 s = {0.0f, 0.0f, 0.0f, 0.0f};
    if (c < a.dim) s = run_share(partial, a.dim, unit, more, c, lane / w, 64 / w);
    for (int off = w; off < 64; off *= 2)
#pragma unroll
      for (int e = 0; e < 4; ++e) s[e] += __shfl_xor(s[e], off);
    if (lane < w && c < a.dim) store(cur, c, s);
  }
  __syncthreads();
  if (s_long < 0) return;  // the same for the block
  const int64_t begin = base + s_long;
  const uint32_t key = keys[(begin + 1) * unit_rows];
  int64_t parts = 0;
  for (;;) {
    const int64_t q = (begin + 1 + parts + tid) * unit_rows;
    const int here = __syncthreads_count(q < a.n && keys[q] == key);
    parts += here;
    if (here < kJoinThreads) break;
  }
  s_sum[tid] = c < a.dim ? run_share(partial, a.dim, begin, parts, c, tid / w, kJoinThreads / w)
                         : f32x4{0.0f, 0.0f, 0.0f, 0.0f};
  __syncthreads();
  for (int g = kJoinThreads / w / 2; g > 0; g /= 2) {
    if (tid < g * w) s_sum[tid] += s_sum[tid + g * w];
    __syncthreads();
  }
  if (tid < w && c < a.dim) store(key, c, s_sum[tid]);
}

// Sorted positions per unit: enough threads (one per 16 bytes of a unit's
// rows) to fill the card, units long enough that few runs cross them.
int unit_rows_for(int64_t n, int64_t dim) {
  int r = kMinUnit;
  while (r < kMaxUnit && n * ceil_div64(dim, 8) / r > kUnitThreads) r *= 2;
  return r;
}

int bits_for(int64_t v) {  // bits of the largest key v
  int b = 1;
  while ((int64_t(1) << b) <= v) ++b;
  return b;
}

int lanes_per_unit(int64_t dim, int elements) { return int(std::min<int64_t>(ceil_div64(dim, elements), kThreads)); }
int units_per_block(int64_t dim, int elements) { return kThreads / lanes_per_unit(dim, elements); }

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
  L.radix = take(radix_ids_tmp_bytes(n));
  // blocks hold the fewest units with the fewest elements per thread, a float's four
  const int64_t blocks = ceil_div64(n, int64_t(unit_rows_for(n, dim)) * units_per_block(dim, 4));
  L.partial = take(size_t(blocks) * 2 * size_t(dim) * 4);
  L.total = off;
  return L;
}

template <typename T>
hipError_t lookup(const EmbeddingArgs& a, hipStream_t s) {
  if (a.n <= 0 || a.dim <= 0) return hipSuccess;
  const int packs = int(ceil_div64(a.dim, Pack<T>::N)), lanes = std::min(packs, kThreads), rpb = kThreads / lanes;
  const int64_t blocks = std::min<int64_t>(ceil_div64(a.n, int64_t(rpb) * kRowsPerThread), 1 << 20);
  // Outputs that the caches would not keep go past them: written through, they
  // push the table out (1M rows of 48 f32: 60 us, past them 38).
  const bool past = a.n * a.dim * int64_t(sizeof(T)) > kCached;
  auto run = [&](auto id) {
    using Id = decltype(id);
    if (past)
      lookup_kernel<T, Id, true><<<uint32_t(blocks), kThreads, 0, s>>>(a, packs, lanes, rpb);
    else
      lookup_kernel<T, Id, false><<<uint32_t(blocks), kThreads, 0, s>>>(a, packs, lanes, rpb);
  };
  if (a.ids64)
    run(int64_t(0));
  else
    run(int32_t(0));
  return hipGetLastError();
}

template <typename T>
hipError_t gradient(const EmbeddingArgs& a, hipStream_t s) {
  if (a.vocab <= 0 || a.dim <= 0) return hipSuccess;
  const int packs = int(ceil_div64(a.dim, Pack<T>::N)), lanes = lanes_per_unit(a.dim, Pack<T>::N);
  const int upb = units_per_block(a.dim, Pack<T>::N);
  const int64_t table_packs = ceil_div64(a.vocab * ceil_div64(a.dim, Pack<T>::N), 4);  // four a thread
  const GradLayout L = grad_layout(a.n, a.dim);
  char* base = static_cast<char*>(a.scratch);
  auto words = [&](size_t off) { return reinterpret_cast<uint32_t*>(base + off); };
  uint32_t *keys = words(L.keys), *pos = words(L.pos);
  const int bits = bits_for(a.vocab);
  hipError_t e;
  if (a.n > 0 && a.n <= kSmallPairs) {
    const uint32_t blocks = uint32_t(1 + std::min<int64_t>(ceil_div64(table_packs, kSmallThreads), 2048));
    if (a.ids64)
      sort_and_zero_kernel<T, int64_t><<<blocks, kSmallThreads, 0, s>>>(a, keys, pos, bits);
    else
      sort_and_zero_kernel<T, int32_t><<<blocks, kSmallThreads, 0, s>>>(a, keys, pos, bits);
    e = hipGetLastError();
  } else {
    const int counting = int(id_sort_blocks(a.n));
    const uint32_t blocks = uint32_t(counting + std::min<int64_t>(ceil_div64(table_packs, kThreads), 8192));
    uint32_t* counts = a.n > 0 ? words(L.radix) : nullptr;
    if (a.ids64)
      count_and_zero_kernel<T, int64_t><<<blocks, kThreads, 0, s>>>(a, counts, counting, id_counts_by_block(a.n));
    else
      count_and_zero_kernel<T, int32_t><<<blocks, kThreads, 0, s>>>(a, counts, counting, id_counts_by_block(a.n));
    e = hipGetLastError();
    if (e != hipSuccess || a.n <= 0) return e;
    e = radix_sort_ids(a.ids, a.ids64, a.vocab, keys, pos, words(L.keys_alt), words(L.pos_alt), a.n, bits,
                       base + L.radix, s);
  }
  if (e != hipSuccess) return e;
  float* partial = reinterpret_cast<float*>(base + L.partial);
  const int unit_rows = unit_rows_for(a.n, a.dim);
  const int block_rows = unit_rows * upb;
  const int64_t blocks = ceil_div64(a.n, block_rows);
  unit_sums_kernel<T><<<uint32_t(blocks), kThreads, 0, s>>>(a, keys, pos, partial, unit_rows, packs, lanes, upb);
  if ((e = hipGetLastError()) != hipSuccess) return e;
  if (blocks > 1)
    join_kernel<T><<<dim3(uint32_t(ceil_div64(blocks, kJoinWaves)), uint32_t(ceil_div64(a.dim, kJoinColumns))),
                     kJoinThreads, 0, s>>>(a, keys, partial, block_rows, blocks);
  return hipGetLastError();
}

}  // namespace

size_t embedding_scratch_bytes(int64_t n, int64_t vocab, int64_t dim) {
  return n > 0 && vocab > 0 && dim > 0 ? grad_layout(n, dim).total : 0;
}

bool embedding_backward_launchable(int64_t n, int64_t dim, gart_dtype t) {
  if (n <= 0 || dim <= 0) return true;
  const int64_t rows = int64_t(unit_rows_for(n, dim)) * units_per_block(dim, 16 / int(dtype_bytes(t)));
  return ceil_div64(n, rows) < (int64_t(1) << 32) / kThreads;
}

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
