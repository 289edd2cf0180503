"""Orthogonalised matrices and momentum steps on the GPU at sizes whose products take the large tiles, with sums whole
and in parts, against plain 64-bit forms."""
import numpy as np
import pytest

import muon_ref as ref
import test_gpu_muon as plain
from muon_sizes import SIZES
from test_gpu_blocks import TYPES, _scratch, _within
from test_gpu_muon import _device, _exact_as_float32, _gradient, _muon_h, _orthogonalize

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


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("rows,cols", AT)
@pytest.mark.parametrize("nesterov,pad,scale", [(True, 0, 1.0), (False, 3, 1.7)])
def test_muon_step(rows, cols, dtype, nesterov, pad, scale):
    plain.test_muon_step(rows, cols, dtype, nesterov, pad, scale)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("rows,cols", [(48, 64), (300, 200), (500, 1500), (960, 2560), (2560, 960)])
def test_muon_leaves_the_gradient(rows, cols, dtype):
    import torch
    from paper_2608_17298_amd import gart
    rng = np.random.default_rng(6)
    p, g = (_device(_gradient(rng, rows, cols), dtype, 3)[0] for _ in range(2))
    m = _device(_gradient(rng, rows, cols), "f32")[0]
    before = g.clone()
    gart.gart_muon_step(p, g, m, _muon_h(gart, 1.0, True), _scratch(gart.gart_muon_scratch_bytes(rows, cols, p.dtype)))
    assert torch.equal(g, before)


@pytest.mark.parametrize("rows,cols,pad", [(960, 2560, 3), (2560, 960, 8), (1472, 1472, 0), (4090, 390, 1), (1000, 1100, 3)])
def test_uses_nothing_around_its_inputs(rows, cols, pad):
    plain.test_uses_nothing_around_its_inputs(rows, cols, pad, "bf16")


@pytest.mark.parametrize("value", [float("nan"), float("inf")])
@pytest.mark.parametrize("rows,cols", [(960, 2560), (2560, 960), (1930, 1921), (450, 3072)])
def test_nonfinite(rows, cols, value):
    plain.test_nonfinite(rows, cols, value, "f32")


@pytest.mark.parametrize("rows,cols", [(1000, 2700), (2560, 960), (1930, 1921)])
def test_another_stream_and_graphs(rows, cols):
    plain.test_another_stream_and_graphs(rows, cols)


@pytest.mark.parametrize("abc", [(3.0, -2.9, 1e-17), (3.0, -3.0, -1e-20), (2.0, -1.9, 1e-30), (-2.0, 1e-25, 2.0)])
@pytest.mark.parametrize("rows,cols", [(2, 5), (20, 30), (70, 300), (300, 200), (500, 700)])
@pytest.mark.parametrize("size", [1.0, 1e-9])
def test_polynomials_with_a_small_coefficient(rows, cols, size, abc):
    """Two singular values of 0.7, in an element each, which the polynomial takes past 1 where the largest of its values
    lies; and, with eps as large, smaller ones."""
    x = np.zeros((rows, cols))
    x[0, 0] = x[1, cols - 1] = size
    t, x64 = _device(x, "f32")
    got = _orthogonalize(t, "f32", steps=3, abc=abc)
    assert np.isfinite(got).all()
    _exact_as_float32(got, x64, "f32", steps=3, abc=[float(np.float32(v)) for v in abc])


@pytest.mark.parametrize("abc", [(0.0, 1.5, -0.5), (1e-20, 1.5, -0.5)])
@pytest.mark.parametrize("rows,cols", [(20, 30), (70, 300), (300, 200)])
@pytest.mark.parametrize("size", [1e-13, 1e-18, 1e-19])
def test_small_matrices_where_the_linear_term_is_small(rows, cols, size, abc):
    """A matrix far smaller than eps, whose a X does not hide what P X has lost."""
    rng = np.random.default_rng(rows)
    x, x64 = _device(rng.standard_normal((rows, cols)) * size / (rows * cols) ** 0.5, "f32")
    _exact_as_float32(_orthogonalize(x, "f32", steps=1, abc=abc), x64, "f32", steps=1,
                      abc=[float(np.float32(v)) for v in abc])
