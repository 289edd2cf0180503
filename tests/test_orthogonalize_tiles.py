"""Which tiles the orthogonalising products are cut into, and who stores them, asked of the C++ rules themselves."""
import os
import subprocess

import pytest

import muon_sizes
import test_gpu_muon

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


CUTS = """
int main() {
  long long rows, cols;
  while (std::scanf("%lld %lld", &rows, &cols) == 2) {
    const MatrixPlan p = matrix_plan(rows, cols);
    const int64_t n = p.n_pad, m = p.m_pad;
    const PairCut c[4] = {cut_pair(n, n, m / 32, true), cut_pair(n, n, n / 32, true), cut_pair(n, m, n / 32, false),
                          p.tall ? cut_pair(m, n, n / 32, false) : cut_pair(n, m, n / 32, false)};
    for (const PairCut& q : c) std::printf("%d %d ", q.side, q.parts);
    std::printf("\\n");
  }
}
"""


def _cuts(tmp_path, sizes):
    """of each size, by product: the tile's side, and whether the sums are cut into parts"""
    return [[(v[2 * k], v[2 * k + 1] > 1) for k in range(4)] for v in _ask(tmp_path, CUTS, sizes)]


def test_every_tile_is_reached_on_the_gpu(tmp_path):
    """The tests' sizes take the tiles that they are listed for, and among them are all that any size takes."""
    listed = _cuts(tmp_path, [s[:2] for s in muon_sizes.SIZES])
    for (rows, cols, want), got in zip(muon_sizes.SIZES, listed):
        assert tuple(got) == (*want, want[2]), (rows, cols)
    steps = range(64, 2200, 64)
    every = [(n, m) for n in steps for m in (*steps, *range(2240, 6000, 256), 20000, 100000)]
    every += [(m, n) for n, m in every]
    reached = {(k, rows > cols, *c) for (rows, cols), q in zip(test_gpu_muon.SIZES + [s[:2] for s in muon_sizes.SIZES],
                                                                _cuts(tmp_path, test_gpu_muon.SIZES) + listed)
               for k, c in enumerate(q)}
    some = {(k, rows > cols, *c) for (rows, cols), q in zip(every, _cuts(tmp_path, every)) for k, c in enumerate(q)}
    # A's and P's products do not know which way x lies
    one_way = lambda s: {c if c[0] > 1 else (c[0], False, *c[2:]) for c in s}  # noqa: E731
    assert one_way(some) <= one_way(reached), one_way(some) - one_way(reached)
