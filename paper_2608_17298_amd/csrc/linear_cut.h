// How a product that does not stream is cut into tiles and parts.  Plain C++, so
// that it can be asked without a GPU.
#pragma once

#include <algorithm>
#include <cstdint>

namespace gart {

// Tiles of 256 (one block of 8 waves a CU, straight into LDS) where they fill the
// card, else of 128, else of 64, and 128 x 32 or 32 x 128 for narrow ones; where
// tiles are few, the sums are cut into parts, which are joined afterwards.
struct Cut {
  int rows, cols;  // of a tile
  int64_t part, parts;
};
constexpr int64_t kJoinParts = 16;      // most parts of y, dz and g_x, whose join has an epilogue
constexpr int64_t kWeightParts = 1024;  // of g_weight

inline int64_t cut_up(int64_t a, int64_t b) { return (a + b - 1) / b; }

// most: parts at most; wide: alignment and sizes allow tiles of 256
inline Cut cut_product(int64_t rows, int64_t cols, int64_t depth, int64_t most, bool wide) {
  constexpr int64_t kCus = 256;
  auto tiles = [&](int i, int j) { return cut_up(rows, i) * cut_up(cols, j); };
  auto parts = [&](int i, int j, int64_t least) {  // two blocks a CU, `least` terms a part
    return std::max<int64_t>(1, std::min({most, 2 * kCus / tiles(i, j), depth / least}));
  };
  auto with = [&](int i, int j, int64_t n) {
    const int64_t part = std::max<int64_t>(64, cut_up(cut_up(depth, n), 64) * 64);
    return Cut{i, j, part, std::max<int64_t>(1, cut_up(depth, part))};
  };
  // Narrow products are bound by their one large operand.
  if (cols <= 32 && rows > 64) return with(128, 32, parts(128, 32, 256));
  if (rows <= 32 && cols > 64) return with(32, 128, parts(32, 128, 256));
  // Up to 128 rows or columns leave half of a tile of 256 empty (60000 x 1024 ->
  // 128 bf16: 37 us, with 128 33; 100000 x 512 -> 16: 38 and, in narrow tiles, 20).
  if (wide && std::min(rows, cols) > 128 && tiles(256, 256) >= kCus * 7 / 8) return with(256, 256, 1);
  // Short sums are bound by their outputs: many small blocks overlap more of
  // them (with 64 and with 128, f32: 20000 x 200 -> 500 53 us and 69, 20000 x 256 ->
  // 500 54 and 71; f16: 20000 x 250 -> 400 19 and 21, 5000 x 256 -> 1024 11 both, but
  // 20000 x 250 -> 1024 46 and 41, 60000 x 100 -> 2300 186 and 162).
  if (depth <= 256) return with(64, 64, 1);
  if (tiles(128, 128) >= kCus * 3 / 2) return with(128, 128, 1);
  // Fewer of 128 leave CUs with one block and nothing to overlap (2000 x 2048 ->
  // 2000 f16: 45 us, in two parts 43, with 64 38); long sums are worth the parts.
  if (tiles(64, 64) >= kCus * 2 && depth <= 4096) return with(64, 64, 1);
  const int64_t p = parts(128, 128, 512);
  return tiles(128, 128) * p >= kCus * 3 / 2 ? with(128, 128, p) : with(64, 64, parts(64, 64, 256));
}

}  // namespace gart
