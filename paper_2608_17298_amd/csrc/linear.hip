// The linear layer's calls: which kernels a size takes, their scratch, and the
// dispatch by element type.
#include <algorithm>

#include "linear_shapes.h"

namespace gart {

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
  if (act != GART_ACT_NONE && !few_rows(m, k, n, es)) cut(m, n, k, kJoinParts);
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
  if (m <= 0 || n <= 0 || few_rows(m, k, n, dtype_bytes(t)) || stream_forward_fits(k, n, dtype_bytes(t))) return 0;
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
  if (few_rows(a.m, a.k, a.n, sizeof(T))) return rows_forward<T>(a, s);
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
