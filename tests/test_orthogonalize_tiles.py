"""Which tiles the orthogonalising products are cut into, and who stores them, asked of the C++ rules themselves."""
import os
import subprocess

import pytest

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2608_17298_amd", "csrc")


def _ask(tmp_path, main, queries):
    src, exe = tmp_path / "tiles.cpp", tmp_path / "tiles"
    src.write_text("#include <cstdio>\n#include <vector>\n" + '#include "orthogonalize.h"\nusing namespace gart;\n' + main)
    subprocess.run(["g++", "-std=c++17", "-O1", "-Wall", "-Werror", "-I", CSRC, str(src), "-o", str(exe)], check=True)
    text = "\n".join(" ".join(str(int(v)) for v in q) for q in queries)
    out = subprocess.run([str(exe)], input=text, check=True, capture_output=True, text=True).stdout
    return [tuple(int(v) for v in line.split()) for line in out.splitlines()]


WRITERS = """
int main() {
  long long rows, cols;
  int side, symmetric;
  while (std::scanf("%lld %lld %d %d", &rows, &cols, &side, &symmetric) == 4) {
    const TileOrder o = tile_order(rows, cols, side, symmetric != 0);
    const int wave = side < 64 ? side : 64;  // what one wave stores, or the waves that split its sums
    const int64_t down = rows / wave, along = cols / wave;
    std::vector<int> writers(down * along);
    for (int t = 0; t < blocks_of(rows, cols, side, symmetric != 0); ++t) {
      int ti, tj;
      if (!find_tile(o, t, ti, tj)) continue;
      for (int i = 0; i < side / wave; ++i)
        for (int j = 0; j < side / wave; ++j) {
          const int64_t i0 = int64_t(ti) * side + i * wave, j0 = int64_t(tj) * side + j * wave;
          if (!is_result(o, rows, cols, i0, j0)) continue;
          ++writers.at(i0 / wave * along + j0 / wave);
          if (symmetric && i0 != j0) ++writers.at(j0 / wave * along + i0 / wave);
        }
    }
    int least = 1 << 30, most = 0;
    for (int w : writers) {
      least = w < least ? w : least;
      most = w > most ? w : most;
    }
    std::printf("%d %d\\n", least, most);
  }
}
"""


@pytest.mark.parametrize("side", [32, 64, 128])
def test_every_block_of_a_product_has_one_writer(tmp_path, side):
    """Also those of a symmetric one, whose blocks above the diagonal are stored on both sides of it: two waves that
    store a block differ in the last bits, and which of them is last would be left to chance."""
    square = [(64 * n, 64 * n, side, 1) for n in range(1, 40)]
    any_size = [(64 * n, 64 * m, side, 0) for n in (1, 2, 3, 7, 16, 33) for m in (1, 2, 5, 8, 31, 200)]
    for q, got in zip(square + any_size, _ask(tmp_path, WRITERS, square + any_size)):
        assert got == (1, 1), q


ORDER = """
int main() {
  long long rows, cols;
  int side, symmetric;
  while (std::scanf("%lld %lld %d %d", &rows, &cols, &side, &symmetric) == 4) {
    const TileOrder o = tile_order(rows, cols, side, symmetric != 0);
    std::printf("%d %d %d\\n", o.tiles_i, o.tiles_j, o.band);
  }
}
"""


def test_order_of_the_most_tiles_stays_in_32_bits(tmp_path):
    """Up to 2^23 tiles of 64 x 64 in all, in one row of tiles as well: what find_tile multiplies fits an int."""
    queries = [(64 * n, 64 * (2 ** 23 // n), side, 0) for n in (1, 2, 3, 5, 64, 2896, 2 ** 22, 2 ** 23)
               for side in (32, 64, 128)]
    queries += [(64 * n, 64 * n, side, 1) for n in (1, 2, 63, 1000, 2896) for side in (32, 64, 128)]
    for q, (i, j, band) in zip(queries, _ask(tmp_path, ORDER, queries)):
        rows, cols = ((i + i % 2) // 2, i + i % 2 + 1) if q[3] else (i, j)
        assert 1 <= band <= rows and rows * cols < 2 ** 31 and band * cols < 2 ** 31, q
