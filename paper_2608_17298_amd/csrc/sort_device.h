// Device code of the sorts, for kernels that sort or count beside other work.
#pragma once

#include <hip/hip_runtime.h>

#include <cstdint>

namespace gart {

constexpr int kSmallThreads = 1024;
constexpr int kSmallWaves = kSmallThreads / 64;
constexpr int64_t kSmallPairs = kSmallThreads * 8;

// Keys and values as they stand in memory.
struct PairSource {
  const uint32_t *keys, *vals;
  __device__ __forceinline__ uint32_t key(int64_t j) const { return keys[j]; }
  __device__ __forceinline__ uint32_t val(int64_t j) const { return vals[j]; }
};

// Ids and their positions; ids outside [0, limit) are sorted last, as limit.
template <typename Id>
struct IdSource {
  const Id* ids;
  int64_t limit;
  __device__ __forceinline__ uint32_t key(int64_t j) const {
    const int64_t id = int64_t(ids[j]);
    return uint32_t(id >= 0 && id < limit ? id : limit);
  }
  __device__ __forceinline__ uint32_t val(int64_t j) const { return uint32_t(j); }
};

// Threads of the device-wide passes.
constexpr int kSortThreads = 256;
// Of a sort of ids, keys per thread: up to a few million, more blocks beat
// longer ones (gradient of 1M ids: 16 keys 147 us, 8 143).
constexpr int kIdItems = 8;
constexpr int64_t kFewBlocks = 128;  // blocks up to which the scatter adds up counts itself

inline int64_t id_sort_blocks(int64_t m) { return (m + kSortThreads * kIdItems - 1) / (kSortThreads * kIdItems); }
inline bool id_counts_by_block(int64_t m) { return id_sort_blocks(m) <= kFewBlocks; }

// Digit counts of one block's keys: counts lie [digit][block], or by block.
template <int ITEMS, typename Source>
__device__ __forceinline__ void radix_count(const Source& source, int64_t m, int shift, uint32_t* __restrict__ counts,
                                            int nblocks, bool by_block) {
  __shared__ uint32_t h[256];
  h[threadIdx.x] = 0;
  __syncthreads();
  const int64_t base = int64_t(blockIdx.x) * (kSortThreads * ITEMS);
  uint32_t kv[ITEMS];
#pragma unroll
  for (int r = 0; r < ITEMS; ++r) {
    const int64_t j = base + int64_t(r) * kSortThreads + threadIdx.x;
    kv[r] = j < m ? source.key(j) : 0u;
  }
#pragma unroll
  for (int r = 0; r < ITEMS; ++r) {
    const int64_t j = base + int64_t(r) * kSortThreads + threadIdx.x;
    if (j < m) atomicAdd(&h[(kv[r] >> shift) & 255u], 1u);
  }
  __syncthreads();
  counts[by_block ? int64_t(blockIdx.x) * 256 + threadIdx.x : int64_t(threadIdx.x) * nblocks + blockIdx.x] =
      h[threadIdx.x];
}

// The valid lanes of the wave whose 8-bit digit is this lane's.  Each bit's
// ballot is matched as ballot == bit in both halves, three operands an instruction.
__device__ __forceinline__ uint64_t same_digit(bool valid, uint32_t d) {
  const uint64_t all = __ballot(valid);
  uint32_t lo = uint32_t(all), hi = uint32_t(all >> 32);
#pragma unroll
  for (int b = 0; b < 8; ++b) {
    const uint32_t bit = uint32_t(int32_t(d << (31 - b)) >> 31);  // all ones or none
    const uint64_t set = __ballot(bit != 0u);
    lo &= ~(uint32_t(set) ^ bit);
    hi &= ~(uint32_t(set >> 32) ^ bit);
  }
  return uint64_t(hi) << 32 | lo;
}

// source.key(j), source.val(j): the pairs to sort, j < m <= kSmallThreads *
// ITEMS, by one block of kSmallThreads threads.  They may lie in keys and vals
// themselves (no restrict): all are read before any is written.
template <int ITEMS, typename Source>
__device__ __forceinline__ void radix_small(const Source& source, uint32_t* keys, uint32_t* vals, int m, int bits) {
  __shared__ uint32_t s_keys[kSmallThreads * ITEMS];
  __shared__ uint32_t s_vals[kSmallThreads * ITEMS];
  __shared__ uint32_t s_wave[kSmallWaves][256];
  __shared__ uint32_t s_wsum[4];
  const int tid = threadIdx.x, wave = tid / 64;
  const unsigned lane = __lane_id();
  const uint64_t lt_mask = (lane == 0) ? 0ull : (~0ull >> (64 - lane));
  const int wbase = wave * 64 * ITEMS;  // this wave's keys: order is wave, round, lane
  uint32_t myk[ITEMS], myv[ITEMS], myr[ITEMS];
#pragma unroll
  for (int r = 0; r < ITEMS; ++r) {
    const int j = wbase + r * 64 + int(lane);
    myk[r] = j < m ? source.key(j) : 0u;
    myv[r] = j < m ? source.val(j) : 0u;
  }
  for (int shift = 0; shift < bits; shift += 8) {
#pragma unroll
    for (int w = 0; w < kSmallWaves / 4; ++w) s_wave[4 * w + tid / 256][tid % 256] = 0;
    __syncthreads();
    volatile uint32_t* wcount = s_wave[wave];
#pragma unroll
    for (int r = 0; r < ITEMS; ++r) {
      if (wbase + r * 64 >= m) break;
      const bool valid = wbase + r * 64 + int(lane) < m;
      const uint32_t d = (myk[r] >> shift) & 255u;
      const uint64_t peers = same_digit(valid, d);
      const uint32_t below = __popcll(peers & lt_mask);
      const uint32_t before = wcount[d];
      myr[r] = before + below;
      if (valid && below == 0) wcount[d] = before + uint32_t(__popcll(peers));
    }
    __syncthreads();
    // digit tid (first 256 threads): start over digits, then each wave's base
    uint32_t total = 0, inc = 0;
    if (tid < 256) {
#pragma unroll
      for (int w = 0; w < kSmallWaves; ++w) total += s_wave[w][tid];
      inc = total;
#pragma unroll
      for (int off = 1; off < 64; off <<= 1) {
        const uint32_t u = __shfl_up(inc, off);
        if (lane >= unsigned(off)) inc += u;
      }
      if (lane == 63) s_wsum[wave] = inc;
    }
    __syncthreads();
    if (tid < 256) {
      uint32_t run = inc - total;
      for (int w = 0; w < wave; ++w) run += s_wsum[w];
#pragma unroll
      for (int w = 0; w < kSmallWaves; ++w) {
        const uint32_t c = s_wave[w][tid];
        s_wave[w][tid] = run;
        run += c;
      }
    }
    __syncthreads();
#pragma unroll
    for (int r = 0; r < ITEMS; ++r) {
      if (wbase + r * 64 + int(lane) < m) {
        const uint32_t pos = s_wave[wave][(myk[r] >> shift) & 255u] + myr[r];
        s_keys[pos] = myk[r];
        s_vals[pos] = myv[r];
      }
    }
    __syncthreads();
#pragma unroll
    for (int r = 0; r < ITEMS; ++r) {
      const int j = wbase + r * 64 + int(lane);
      myk[r] = j < m ? s_keys[j] : 0u;
      myv[r] = j < m ? s_vals[j] : 0u;
    }
  }
#pragma unroll
  for (int r = 0; r < ITEMS; ++r) {
    const int j = wbase + r * 64 + int(lane);
    if (j < m) {
      keys[j] = myk[r];
      vals[j] = myv[r];
    }
  }
}

}  // namespace gart
