"""The linear layer's tiled products at sizes that take every tile, whole and cut into parts, with several steps of
the sum (linear_sizes.py; test_linear_cut.py asserts the tiles)."""
import numpy as np
import pytest

import blocks_ref as ref
import linear_sizes as ls
from test_gpu_blocks import _Out, _integers, _mat, _rounded, _scratch, _torch, _vec, _within
from test_gpu_linear_gradient import _gradients, _tolerance

pytestmark = pytest.mark.gpu

CASES = [(m, k, n, pad, d) for m, k, n, pad, dtypes, _ in ls.SIZES for d in dtypes]


@pytest.mark.parametrize("m,k,n,pad,dtype", CASES)
def test_tiles_are_exact_in_whole_numbers(m, k, n, pad, dtype):
    """Whole numbers whose sums stay below 2^24: every sum is exact in float, in any order, so each result is the
    exact one rounded once.  relu with half-integer biases decides every slope exactly."""
    from paper_2608_17298_amd import gart
    rng = np.random.default_rng(m + 2 * k + 3 * n)
    x, x64 = _integers(rng, m, k, dtype, pad, 1)
    w, w64 = _integers(rng, n, k, dtype, pad, 2)
    dl, d64 = _integers(rng, m, n, dtype, pad, 2)
    b, b64 = _integers(rng, 1, n, dtype, 0, 3)
    b, b64 = (b[0] + 0.5).contiguous(), b64[0] + 0.5
    x32, w32, t = x64.astype(np.float32), w64.astype(np.float32), _torch(dtype)
    y = _Out(m, n, dtype, pad)
    gart.gart_linear(x, w, y.t, b, None, "relu", _scratch(gart.gart_linear_scratch_bytes(m, k, n, t)))
    z = (x32 @ w32.T).astype(np.float64) + b64
    assert np.array_equal(y.value(), _rounded(np.maximum(z, 0.0), dtype))
    for act in ("relu", "none"):
        dz = (np.where(z > 0, d64, 0.0) if act == "relu" else d64).astype(np.float32)
        want = (dz @ w32, dz.T @ x32, dz.sum(axis=0, dtype=np.float64))
        for got, a in zip(_gradients(x, w, dl, b, act, dtype, pad), want):
            assert np.abs(a).max() < 60000  # float16 holds it
            assert np.array_equal(got, _rounded(a.astype(np.float64), dtype))


@pytest.mark.parametrize("m,k,n,pad,dtype", [c for c in CASES if c[4] != "f32"])
def test_tiles_with_dz_in_two_parts(m, k, n, pad, dtype):
    """The same tiles for silu, whose dz is high + low: the low parts come in the right places and with their scale."""
    rng = np.random.default_rng(m + 5 * k + 7 * n)
    (x, x64), (w, w64) = _mat(rng, m, k, dtype, pad), _mat(rng, n, k, dtype, pad, k ** -0.5)
    (b, b64), (dl, d64) = _vec(rng, n, dtype), _mat(rng, m, n, dtype, pad)
    got = _gradients(x, w, dl, b, "silu", dtype, pad)
    tol = _tolerance(x64, w64, b64, d64, "silu", dtype)
    for g, want, q in zip(got, ref.linear_grads(x64, w64, b64, d64, "silu"), tol):
        _within(g, want, q)
