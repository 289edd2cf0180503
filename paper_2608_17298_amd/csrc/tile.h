// One operand's tile of a product in LDS, and the order of tiles over the XCDs.
#pragma once

#include "linear.h"

namespace gart {
namespace {

constexpr int kLine = 128;  // bytes of k per step

template <typename T>
constexpr int kStep = kLine / int(sizeof(T));  // k per step

// One operand's tile of ROWS rows (i) and kStep columns (k) in LDS.  PERM: the
// rows a fragment takes are the output's j, paired up (paired_row).
template <typename T, bool KC, int ROWS, int WAVES, bool PERM>
struct Tile {
  static constexpr int V = Pack<T>::N, THREADS = 64 * WAVES;
  static constexpr bool SHORT = sizeof(T) == 2;
  // float lines are padded instead: a fragment reads single elements of four lines
  static constexpr int PITCH = KC ? kStep<T> : SHORT ? ROWS : ROWS + 4;
  static constexpr int LINE_PACKS = KC ? kStep<T> / V : ROWS / V;  // packs per line in memory
  static constexpr int LINES = KC ? ROWS : kStep<T>;
  static constexpr int ELEMS = LINES * PITCH;
  static constexpr int PACKS = LINES * LINE_PACKS;
  static constexpr int PER_THREAD = PACKS / THREADS;
  static_assert(PACKS % THREADS == 0, "whole packs per thread");

  // Exchange of a line's 16-byte pieces: distinct pieces for any eight rows that
  // are read together; pairs of pieces for the lines 0-3 and 8-11 of columns.
  static __device__ __forceinline__ int swizzle(int line) {
    if (KC) return PERM && SHORT ? (line & 3) | ((line >> 1) & 4) : line & 7;
    if (!SHORT) return 0;
    return 2 * (ROWS >= 128  ? (line & 3) | ((line >> 1) & 4)
                : ROWS >= 64 ? ((line >> 1) & 1) | ((line >> 2) & 2)
                             : (line >> 3) & 1);
  }

  // ---- through registers: any size and alignment ----
  // rows x ks elements are there; i0, k0: where the tile begins
  static __device__ __forceinline__ void load_edge(Pack<T> (&reg)[PER_THREAD], const T* __restrict__ p, int64_t ld,
                                                   int64_t i0, int64_t rows, int64_t k0, int64_t ks, int tid) {
#pragma unroll
    for (int u = 0; u < PER_THREAD; ++u) {
      const int c = u * THREADS + tid;
      const int line = c / LINE_PACKS, at = (c % LINE_PACKS) * V;
      const int64_t l = (KC ? i0 : k0) + line, o = (KC ? k0 : i0) + at;
      const int64_t lines = KC ? rows : ks, length = KC ? ks : rows;
      reg[u].v = T(0.0f);
      if (l < lines && o < length) reg[u] = load_some(p + l * ld + o, int(min(int64_t(V), length - o)));
    }
  }
  static __device__ __forceinline__ void store(T* lds, const Pack<T> (&reg)[PER_THREAD], int tid) {
#pragma unroll
    for (int u = 0; u < PER_THREAD; ++u) {
      const int c = u * THREADS + tid;
      const int line = c / LINE_PACKS, piece = c % LINE_PACKS ^ swizzle(line);
      *reinterpret_cast<typename Pack<T>::V*>(lds + line * PITCH + piece * V) = reg[u].v;
    }
  }

  // ---- whole steps of k, without checks ----
  // Rows past the end repeat the last one (pack of them, for lines across k);
  // their products are not stored.  Needs whole packs of rows at the end.
  static __device__ __forceinline__ bool regular(int64_t i0, int64_t rows) {
    return KC || i0 + ROWS <= rows || rows % V == 0;
  }
  const T* from[PER_THREAD];

  // DIRECT: in the order of LDS, where a wave's 64 packs land side by side
  template <bool DIRECT>
  __device__ __forceinline__ void aim(const T* p, int64_t ld, int64_t i0, int64_t rows, int64_t k0, int tid) {
#pragma unroll
    for (int u = 0; u < PER_THREAD; ++u) {
      const int c = u * THREADS + tid;
      const int line = c / LINE_PACKS, at = (DIRECT ? c % LINE_PACKS ^ swizzle(line) : c % LINE_PACKS) * V;
      from[u] = KC ? p + min(i0 + line, rows - 1) * ld + k0 + at : p + (k0 + line) * ld + min(i0 + at, rows - V);
    }
  }
  static __device__ __forceinline__ int64_t stride(int64_t ld) { return KC ? int64_t(kStep<T>) : kStep<T> * ld; }

  __device__ __forceinline__ void load(Pack<T> (&reg)[PER_THREAD], int64_t offset) const {
#pragma unroll
    for (int u = 0; u < PER_THREAD; ++u) reg[u] = load_pack(from[u] + offset);
  }
  __device__ __forceinline__ void fetch(T* lds, int64_t offset, int wave) const {
    typedef const __attribute__((address_space(1))) uint32_t* global_ptr;
    typedef __attribute__((address_space(3))) uint32_t* lds_ptr;
#pragma unroll
    for (int u = 0; u < PER_THREAD; ++u)
      __builtin_amdgcn_global_load_lds((global_ptr)(from[u] + offset),
                                       (lds_ptr)(lds + (u * THREADS + 64 * wave) * V), 16, 0, 0);
  }

  // fragment of 16 rows at tile `tile`, step `s` of the line's two
  static __device__ __forceinline__ typename Pack<T>::V fragment(const T* lds, int tile, int s, int lane) {
    const int r = lane % 16, g = lane / 16;
    if constexpr (KC) {
      const int row = PERM ? paired_row<T>(tile, r) : 16 * tile + r;
      return fragment_of_row(lds, PITCH, row, 0, (4 * s + g) ^ swizzle(row));
    } else if constexpr (!SHORT) {
      return fragment_of_columns(lds, PITCH, tile, kDepth<T> * s, lane);
    } else {
      const int line = kDepth<T> * s + 8 * g + r / 4;  // line + 4 has the same exchange
      const int col = PERM ? paired_row<T>(tile, 4 * (r % 4)) : 16 * tile + 4 * (r % 4);
      return transposed_pair(lds + line * PITCH + ((col / V) ^ swizzle(line)) * V + col % V, 4 * PITCH);
    }
  }
};

// Blocks are dealt to the eight XCDs in turn; each XCD gets a contiguous run of
// tiles, which share rows of A in its L2.
__device__ __forceinline__ int64_t xcd_tile(int64_t b, int64_t total) {
  const int64_t q = total / 8, r = total % 8, x = b % 8;
  return x * q + min(x, r) + b / 8;
}

}  // namespace
}  // namespace gart
