// The linear layer's calls: which kernels a size takes, their scratch, and the
// dispatch by element type.
#include <algorithm>

#include "linear_shapes.h"

namespace gart {

Cut cut_product(int64_t rows, int64_t cols, int64_t depth, int64_t most, bool wide) {
  constexpr int64_t kCus = 256;
  auto tiles = [&](int i, int j) { return ceil_div64(rows, i) * ceil_div64(cols, j); };
  auto parts = [&](int i, int j, int64_t least) {  // two blocks a CU, `least` terms a part
    return std::max<int64_t>(1, std::min({most, 2 * kCus / tiles(i, j), depth / least}));
  };
  auto with = [&](int i, int j, int64_t n) {
    const int64_t part = std::max<int64_t>(64, ceil_div64(ceil_div64(depth, n), 64) * 64);
    return Cut{i, j, part, std::max<int64_t>(1, ceil_div64(depth, part))};
  };
  // Narrow products are bound by their one large operand.
  if (cols <= 32 && rows > 64) return with(128, 32, parts(128, 32, 256));
  if (rows <= 32 && cols > 64) return with(32, 128, parts(32, 128, 256));
  // Up to 128 rows or columns leave half of a tile of 256 empty (60000 x 1024 ->
  // 128 bf16: 37 us, with 128 33; 100000 x 512 -> 16: 38 and, in narrow tiles, 20).
  if (wide && std::min(rows, cols) > 128 && tiles(256, 256) >= kCus * 7 / 8) return with(256, 256, 1);
  // Short sums are bound by their outputs: many small blocks overlap more of
  // them (20000 x 256 -> 1024 f16: 49 us with 128, 44 with 64; 20000 x 200 -> 500
  // f32: 99 and 62; 8000 x 512 -> 1000 f16: 22 and 25).
  if (depth <= 256) return with(64, 64, 1);
  if (tiles(128, 128) >= kCus * 3 / 2) return with(128, 128, 1);
  // Fewer of 128 leave CUs with one block and nothing to overlap (2000 x 2048 ->
  // 2000 f16: 45 us, in two parts 43, with 64 38); long sums are worth the parts.
  if (tiles(64, 64) >= kCus * 2 && depth <= 4096) return with(64, 64, 1);
  const int64_t p = parts(128, 128, 512);
  return tiles(128, 128) * p >= kCus * 3 / 2 ? with(128, 128, p) : with(64, 64, parts(64, 64, 256));
}

// Without inputs there is nothing that a stream could read a pack of.
bool stream_forward_fits(int64_t k, int64_t n, size_t es) {
  return k > 0 && k <= 512 / int64_t(es) && n <= 2048 && forward_lds(round_inputs(k), n, es) <= kForwardBytes;
}

int64_t stream_backward_parts(int64_t m, int64_t k, int64_t n, size_t es) {
  if (m <= 0 || k <= 0 || n <= 0) return 0;
  const BackwardChoice c = choose_backward(k, n, es);
  return c.kp == 0 ? 0 : backward_blocks(ceil_div64(m, c.rows));
}

BackwardPlan backward_plan(int64_t m, int64_t k, int64_t n, gart_dtype t, gart_activation act) {
  BackwardPlan p{};
  const size_t es = dtype_bytes(t);
  size_t off = 0;
  auto take = [&](size_t bytes) {
    const size_t o = off;
    off += (bytes + 255) & ~size_t(255);
    return o;
  };
  auto floats = [](int64_t parts, int64_t rows, int64_t cols) {
    return size_t(parts) * size_t(rows) * size_t(cols) * 4;
  };
  p.parts = stream_backward_parts(m, k, n, es);
  const bool one_block = p.parts == 1 && k <= kSmallStreamInputs && n * k <= kSmallStreamWeight;
  p.small = es == 2 && act != GART_ACT_NONE && m > 0 && n > 0 && k > 0 && k <= kSmallInputs &&
            m * n <= kSmallElements && !one_block;
  if (p.small) {
    p.dz = take(size_t(m * n) * 4);
    p.total = off;
    return p;
  }
  if (p.parts > 0) {
    p.stream = true;
    p.partial = take(p.parts > 1 ? floats(p.parts, n, k + 1) : 0);
    p.total = off;
    return p;
  }
  p.dz_ld = (n + 7) / 8 * 8;
  p.dz_low = dz_in_parts(act, es) ? m * p.dz_ld : 0;
  p.dz = take(act == GART_ACT_NONE ? 0 : size_t(m * p.dz_ld + p.dz_low) * es);
  // Products that are cut leave their parts here, one after the other; tiles of
  // 256 are never cut, and where they could be taken those of 128 are not either.
  size_t parts = 0;
  auto cut = [&](int64_t rows, int64_t cols, int64_t depth, int64_t most) {
    if (rows <= 0 || cols <= 0) return;
    const Cut c = cut_product(rows, cols, depth, most, false);
    if (c.parts > 1) parts = std::max(parts, floats(c.parts, rows, cols));
  };
  if (act != GART_ACT_NONE && !few_rows(m, n)) cut(m, n, k, kJoinParts);
  cut(m, k, n, kJoinParts);
  cut(n, k, m, kWeightParts);
  p.partial = take(parts);
  p.sums = take(floats(std::max<int64_t>(ceil_div64(m, kJoinRows), 1), 1, n));
  p.total = off;
  return p;
}

namespace {

constexpr int64_t kMaxTiles = int64_t(1) << 23;  // blocks of a launch

bool launchable(int64_t rows, int64_t cols) { return ceil_div64(rows, 64) * ceil_div64(cols, 64) <= kMaxTiles; }

}  // namespace

int64_t linear_scratch_bytes(int64_t m, int64_t k, int64_t n, gart_dtype t) {
  if (m <= 0 || n <= 0 || few_rows(m, n) || stream_forward_fits(k, n, dtype_bytes(t))) return 0;
  if (!launchable(m, n)) return -1;
  const Cut c = cut_product(m, n, k, kJoinParts, false);
  return c.parts > 1 ? c.parts * m * n * 4 : 0;
}

int64_t linear_backward_scratch_bytes(int64_t m, int64_t k, int64_t n, gart_dtype t, gart_activation act) {
  if (stream_backward_parts(m, k, n, dtype_bytes(t)) == 0 &&
      !(launchable(m, n) && launchable(m, k) && launchable(n, k) && ceil_div64(n, 64) < 65536))
    return -1;
  return int64_t(backward_plan(m, k, n, t, act).total);
}

namespace {

template <typename T>
hipError_t forward(const LinearArgs& a, hipStream_t s) {
  if (few_rows(a.m, a.n)) return rows_forward<T>(a, s);
  return stream_forward_fits(a.k, a.n, sizeof(T)) ? stream_forward<T>(a, s) : gemm_forward<T>(a, s);
}

}  // namespace

hipError_t launch_linear(const LinearArgs& a, gart_dtype t, hipStream_t s) {
  if (t == GART_DTYPE_F32) return forward<float>(a, s);
  if (t == GART_DTYPE_BF16) return forward<bf16>(a, s);
  return forward<f16>(a, s);
}

hipError_t launch_linear_backward(const LinearArgs& a, gart_dtype t, hipStream_t s) {
  if (t == GART_DTYPE_F32) return gemm_backward<float>(a, s);
  if (t == GART_DTYPE_BF16) return gemm_backward<bf16>(a, s);
  return gemm_backward<f16>(a, s);
}

}  // namespace gart
