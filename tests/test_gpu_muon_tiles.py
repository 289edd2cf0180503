"""Orthogonalised matrices and momentum steps on the GPU at sizes whose products take the large tiles, with sums whole
and in parts, against plain 64-bit forms."""
import numpy as np
import pytest

import muon_ref as ref
from muon_sizes import SIZES
from test_gpu_blocks import TYPES, _within
from test_gpu_muon import _device, _exact_as_float32, _gradient, _orthogonalize

pytestmark = pytest.mark.gpu

AT = [s[:2] for s in SIZES]


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("rows,cols", AT)
def test_same_bits_every_time(rows, cols, dtype):
    rng = np.random.default_rng(rows + cols)
    x, x64 = _device(_gradient(rng, rows, cols), dtype, 3)
    got = [_orthogonalize(x, dtype, 5) for _ in range(4)]
    assert all(np.array_equal(got[0], g) for g in got[1:])
    _exact_as_float32(got[0], x64, dtype)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("rows,cols", AT)
def test_one_step_element_by_element(rows, cols, dtype):
    rng = np.random.default_rng(rows + 5 * cols)
    x, x64 = _device(_gradient(rng, rows, cols, "normal"), dtype, 1)
    _within(_orthogonalize(x, dtype, 3, steps=1), ref.orthogonalize(x64, 1), ref.one_step_tolerance(x64, dtype))
