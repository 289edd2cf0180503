"""Which tiles the linear layer's products take, asked of the C++ rule itself: the GPU tests of every tile do reach it."""
import os
import subprocess

import linear_sizes as ls

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2608_17298_amd", "csrc")

MAIN = """#include <cstdio>
#include "linear_cut.h"
int main() {
  long long q[5];
  while (std::scanf("%lld %lld %lld %lld %lld", q, q + 1, q + 2, q + 3, q + 4) == 5) {
    const gart::Cut c = gart::cut_product(q[0], q[1], q[2], q[3] ? gart::kWeightParts : gart::kJoinParts, q[4] != 0);
    std::printf("%d %d %lld %lld\\n", c.rows, c.cols, (long long)c.part, (long long)c.parts);
  }
}
"""


def _cuts(tmp_path, queries):
    src, exe = tmp_path / "cut.cpp", tmp_path / "cut"
    src.write_text(MAIN)
    subprocess.run(["g++", "-std=c++17", "-O1", "-Wall", "-Werror", "-I", CSRC, str(src), "-o", str(exe)], check=True)
    text = "\n".join(" ".join(str(int(v)) for v in q) for q in queries)
    out = subprocess.run([str(exe)], input=text, check=True, capture_output=True, text=True).stdout
    return [tuple(int(v) for v in line.split()) for line in out.splitlines()]


def _products(m, k, n, pad, dtype):
    """rows, columns, length of the sums, weight's parts allowed, tiles of 256 allowed: y, g_x, g_weight (of dz in
    scratch, whose rows are aligned)."""
    short = dtype != "f32"
    even = (k + pad) % 8 == 0
    return [(m, n, k, 0, short and k % 64 == 0 and even), (m, k, n, 0, short and n % 64 == 0 and even and k % 8 == 0),
            (n, k, m, 1, short and m % 64 == 0 and even and n % 8 == 0 and k % 8 == 0)]


def test_sizes_take_the_tiles_they_are_listed_for(tmp_path):
    want, queries = [], []
    for m, k, n, pad, dtypes, tiles in ls.SIZES:
        for dtype in dtypes:
            for q, tile in zip(_products(m, k, n, pad, dtype), tiles):
                if tile is not None:
                    queries.append(q)
                    want.append(tile)
    got = _cuts(tmp_path, queries)
    for q, w, (rows, cols, _, parts) in zip(queries, want, got):
        assert (rows, cols, parts > 1) == w, q
    assert set(want) == {ls.T256, ls.T128, ls.P128, ls.T64, ls.P64, ls.TALL, ls.TALL_PARTS,
                         ls.FLAT, ls.FLAT_PARTS}
    steps = {q[2] // 64 for q, w in zip(queries, want) if w == ls.T256}
    assert steps == {2, 3, 5}  # even and odd numbers of steps between the two buffers


def test_parts_cover_the_sum(tmp_path):
    queries = [(r, c, d, w, 0) for r in (1, 33, 64, 1000, 5000) for c in (1, 32, 65, 1000) for w in (0, 1)
               for d in (0, 1, 64, 65, 500, 4097, 100000, 2 ** 31 - 1)]
    for (r, c, d, w, _), (rows, cols, part, parts) in zip(queries, _cuts(tmp_path, queries)):
        assert part % 64 == 0 and 1 <= parts <= (1024 if w else 16)
        assert part * parts >= d and (parts == 1 or part * (parts - 1) < d)
