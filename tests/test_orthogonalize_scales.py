"""The scales of the orthogonalising steps' operands, asked of the C++ rule: no polynomial that the call accepts takes
an operand past float16's range."""
import ctypes
import os
import subprocess

import numpy as np
import pytest

import muon_ref as ref

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2608_17298_amd", "csrc")
MAIN = """#include <cstdio>
#include "orthogonalize.h"
int main() {
  double a, b, c, bound;
  int steps;
  while (std::scanf("%lf %lf %lf %lf %d", &a, &b, &c, &bound, &steps) == 5) {
    for (int k = 0; k < steps; ++k) {
      gart::StepScales s;
      bound = gart::step_scales(a, b, c, bound, &s);
      std::printf(" %.17g %.17g %.17g %.17g", s.x, s.a, s.p, bound);
    }
    std::printf("\\n");
  }
}
"""


def _scales(tmp_path, sets, start, steps):
    """[set][step] (scales of X, A and P, bound after the step)"""
    src, exe = tmp_path / "s.cpp", tmp_path / "s"
    src.write_text(MAIN)
    subprocess.run(["g++", "-std=c++17", "-O1", "-Wall", "-Werror", "-I", CSRC, str(src), "-o", str(exe)], check=True)
    text = "\n".join(" ".join(repr(v) for v in (*q, start, steps)) for q in sets)
    out = subprocess.run([str(exe)], input=text, capture_output=True, text=True, check=True).stdout
    return [np.array([float(v) for v in line.split()]).reshape(steps, 4) for line in out.strip().split("\n")]


# polynomials with a small coefficient beside larger ones: the derivative's roots in s^2 are far apart
SMALL = [(3.0, -2.9, 1e-17), (3.0, -3.0, 1e-20), (3.0, -3.0, -1e-20), (2.0, -1.9, 1e-12), (2.0, -1.9, 1e-30),
         (1.5, -0.5, 1e-38), (1e-17, 3.0, -2.9), (-1e-20, 2.0, -2.0), (2.0, 1e-18, -1.9), (2.0, -1e-18, -1.9),
         (-2.0, 1e-25, 2.0), (-3.0, 2.9, 1e-17), (0.0, 1.5, -1e-17), (0.0, -1.0, 1.0), (1e-30, -1.0, 1e-30)]


@pytest.mark.parametrize("start", [1.0, 0.0625, 1e-3])
def test_bounds_hold_where_a_coefficient_is_small(tmp_path, start):
    """Against each polynomial on a fine grid of the interval that the step's values fill: no value passes the bound
    (and it is no more than the grid's own step above the largest), and X stays below 2^14 of its scale's inverse."""
    for (a, b, c), steps in zip(SMALL, _scales(tmp_path, SMALL, start, 6)):
        filled = start
        for x, _, _, bound in steps:
            if filled > 1024.0:  # the call refuses such steps
                break
            s = np.linspace(0.0, filled, 200001)
            reach = np.abs(a * s + b * s ** 3 + c * s ** 5).max()
            assert filled * x <= 2.0 ** 14, (a, b, c)
            # an extremum is 2.5e-6 of the interval from the grid at most, and |p''| is at most 26 times the largest
            # term: the grid's maximum is 8e-11 of that below; a sum of three rounded terms is 1e-15 of it off
            size = max(abs(a) * filled, abs(b) * filled ** 3, abs(c) * filled ** 5)
            assert reach - 1e-14 * size <= bound <= reach + 1e-9 * size, (a, b, c)
            filled = bound


def test_growth_inside_the_interval_is_refused():
    """3000 (s - s^3) is 0 at 1 and 1155 at 0.577: past 1024, with a fifth power of next to nothing as well."""
    from paper_2608_17298_amd import gart
    lib, mb = gart.lib(), 1 << 20
    x, y = (ctypes.byref(gart.gart_matrix(k * mb, 4, 8, 8)) for k in (1, 2))
    need = lib.gart_orthogonalize_scratch_bytes(4, 8, 0)
    for c in (0.0, 1e-16, -1e-16, 1e-38):
        how = gart.gart_newton_schulz(3000.0, -3000.0, c, 1e-7, 1)
        assert lib.gart_orthogonalize(x, ctypes.byref(how), 0, y, 8 * mb, need, None) == -1, c
        assert "1024" in lib.gart_last_error().decode()


FACTORS = """#include <cstdio>
#include "orthogonalize.h"
int main() {
  double a, b, c, bound;
  int steps;
  while (std::scanf("%lf %lf %lf %lf %d", &a, &b, &c, &bound, &steps) == 5) {
    float x;
    gart::StepFactors f[gart::kMaxSteps];
    if (!gart::step_factors(float(a), float(b), float(c), steps, bound, &x, f)) return 1;
    std::printf("%.9g", x);
    for (int k = 0; k < steps; ++k)
      std::printf(" %.9g %.9g %.9g %.9g %.9g", f[k].gram, f[k].square, f[k].linear, f[k].apply, f[k].keep);
    std::printf("\\n");
  }
}
"""


def _pair(v):
    """As the kernels hold it: the sum of two float16 numbers."""
    high = v.astype(np.float32).astype(np.float16)
    low = (v.astype(np.float32) - high.astype(np.float32)).astype(np.float16)
    return high.astype(np.float64) + low.astype(np.float64)


@pytest.mark.parametrize("abc", [(0.0, 1.5, -0.5), (1e-20, 1.5, -0.5), (1e-9, 1.5, 0.0), (0.0, 0.0, 1.0),
                                 (3.4445, -4.775, 2.0315)])
@pytest.mark.parametrize("size", [1e-9, 1e-13, 1e-16, 1e-18, 1e-19, 3e-20])
def test_small_matrices_where_the_linear_term_is_small(tmp_path, abc, size):
    """The kernels' arithmetic with the scales of a matrix far smaller than eps: a result of float32's own range is as
    exact as float32's, also where a X does not hide what is lost in P X."""
    src, exe = tmp_path / "f.cpp", tmp_path / "f"
    src.write_text(FACTORS)
    subprocess.run(["g++", "-std=c++17", "-O1", "-Wall", "-Werror", "-I", CSRC, str(src), "-o", str(exe)], check=True)
    rng = np.random.default_rng(5)
    x = (rng.standard_normal((12, 17)) * size).astype(np.float32).astype(np.float64)
    abc, eps = [float(np.float32(v)) for v in abc], float(np.float32(1e-7))
    norm = np.sqrt((x ** 2).sum())
    out = subprocess.run([str(exe)], input=" ".join(repr(float(v)) for v in (*abc, norm / (norm + eps), 1)),
                         capture_output=True, text=True, check=True).stdout
    first, *f = (np.float32(v) for v in out.split())
    h = _pair(x * (float(first) / (norm + eps)))
    gram, square, linear, apply, keep = f
    q = _pair(gram * (h @ h.T).astype(np.float32))
    p = _pair(linear * q.astype(np.float32) + square * (q @ q).astype(np.float32))
    got = (apply * (p @ h).astype(np.float32) + keep * h.astype(np.float32)).astype(np.float64)
    want = ref.orthogonalize(x, 1, abc, eps)
    # X (five times, in the powers of the formula), A twice and P are off by 2^-22 of an element or less, roundings to
    # float32 by a fourth of that: 10 such of the terms, whose sums are below the products of the norms; and the
    # sums of P X, up to 2^28, are multiplied by a float at last, which is off by 2^-150 where it is that small
    a, b, c = np.abs(abc)
    x /= norm + eps
    q, x = np.linalg.norm(x @ x.T), np.linalg.norm(x)
    assert (np.abs(got - want) <= 10 * 2.0 ** -22 * (a + b * q + c * q * q) * x + 2.0 ** -122).all()
