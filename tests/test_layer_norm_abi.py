"""CPU checks of the layer norm's C ABI: invalid arguments are refused before the device is touched, sizes of scratch,
empty calls, and the 64-bit gradient itself by differences."""
import ctypes

import numpy as np
import pytest

import layer_norm_ref as ref

INVALID = -1
MB = 1 << 20


def _m(gart, addr, rows, cols, stride=None):
    return gart.gart_matrix(addr, rows, cols, cols if stride is None else stride)


def _lib():
    from paper_2608_17298_amd import gart
    return gart, gart.lib()


def _err(lib):
    return lib.gart_last_error().decode()


FORWARD_BAD = dict(
    x_null=("x data", dict(x=(0, 4, 8))), stride=("row stride", dict(x=(MB, 4, 8, 7))),
    negative=("-1", dict(x=(MB, -1, 8))), cols=("differ in size", dict(y=(3 * MB, 4, 9))),
    rows=("differ in size", dict(y=(3 * MB, 5, 8))), y_stride0=("row stride", dict(y=(3 * MB, 4, 8, 0))),
    unaligned=("aligned", dict(x=(MB + 2, 4, 8))), y_overlaps=("overlaps x", dict(y=(MB + 16, 4, 8))),
    y_restrided=("overlaps x", dict(x=(MB, 4, 8, 16), y=(MB, 4, 8, 8))),
    gain=("gain", dict(gain=5 * MB + 1)), bias=("bias", dict(bias=5 * MB + 2)),
    y_is_gain=("gain or bias", dict(gain=3 * MB + 8)), y_is_bias=("gain or bias", dict(bias=3 * MB)),
    dtype=("dtype", dict(dtype=3)), eps=("eps", dict(eps=-1e-9)), eps_nan=("eps", dict(eps=float("nan"))),
    eps_inf=("eps", dict(eps=float("inf"))), too_many=("x is", dict(x=(MB, 1 << 31, 8))))


@pytest.mark.parametrize("name", sorted(FORWARD_BAD))
def test_refusals(name):
    gart, lib = _lib()
    a = dict(x=(MB, 4, 8), y=(3 * MB, 4, 8), gain=None, bias=None, eps=1e-5, dtype=0)
    word, change = FORWARD_BAD[name]
    a.update(change)
    x, y = (ctypes.byref(_m(gart, *a[k])) for k in ("x", "y"))
    r = lib.gart_layer_norm(x, a["gain"], a["bias"], a["eps"], a["dtype"], y, None)
    assert r == INVALID and word in _err(lib), _err(lib)


BACKWARD_BAD = dict(
    dl_rows=("differ in size", dict(dl=(2 * MB, 5000, 8))), dl_cols=("differ in size", dict(dl=(2 * MB, 4000, 7))),
    g_x_size=("g_x and x", dict(g_x=(3 * MB, 4000, 7))), g_x_stride=("row stride", dict(g_x=(3 * MB, 4000, 8, 0))),
    g_x_is_x=("overlaps an input", dict(g_x=(MB, 4000, 8))), g_x_is_dl=("overlaps an input", dict(g_x=(2 * MB, 4000, 8))),
    g_gain_is_gain=("overlaps an input", dict(g_gain=4 * MB)),
    together=("gradients overlap", dict(g_bias=5 * MB + 4)), gain=("gain", dict(gain=4 * MB + 1)),
    g_gain=("g_gain", dict(g_gain=5 * MB + 1)), g_bias=("g_bias", dict(g_bias=6 * MB + 3)),
    eps=("eps", dict(eps=-1.0)), dtype=("dtype", dict(dtype=-1)), no_scratch=("scratch is NULL", dict(scratch=None)),
    short=("scratch_bytes", dict(short=1)), scratch_odd=("16-byte", dict(scratch=9 * MB + 8)),
    **{f"scratch_on_{k}": ("scratch overlaps", dict(scratch=k * MB + 16)) for k in range(1, 7)})


@pytest.mark.parametrize("name", sorted(BACKWARD_BAD))
def test_backward_refusals(name):
    gart, lib = _lib()
    a = dict(x=(MB, 4000, 8), dl=(2 * MB, 4000, 8), g_x=(3 * MB, 4000, 8), gain=4 * MB, g_gain=5 * MB, g_bias=6 * MB, eps=1e-5,
             dtype=0, scratch=9 * MB, short=0)
    word, change = BACKWARD_BAD[name]
    a.update(change)
    x, dl, g_x = (ctypes.byref(_m(gart, *a[k])) for k in ("x", "dl", "g_x"))
    need = lib.gart_layer_norm_backward_scratch_bytes(4000, 8, 0)
    assert 0 < need < MB
    r = lib.gart_layer_norm_backward(x, dl, a["gain"], a["eps"], a["dtype"], g_x, a["g_gain"], a["g_bias"],
                                     a["scratch"], need - a["short"], None)
    assert r == INVALID and word in _err(lib), _err(lib)


def test_null_matrices_refused():
    gart, lib = _lib()
    x = ctypes.byref(_m(gart, MB, 4, 8))
    assert lib.gart_layer_norm(None, None, None, 1e-5, 0, x, None) == INVALID
    assert lib.gart_layer_norm(x, None, None, 1e-5, 0, None, None) == INVALID
    assert lib.gart_layer_norm_backward(None, x, None, 1e-5, 0, None, None, None, None, 0, None) == INVALID
    assert lib.gart_layer_norm_backward(x, None, None, 1e-5, 0, None, None, None, None, 0, None) == INVALID


def test_empty_calls_need_nothing():
    """No rows or no columns: nothing is launched, whatever the pointers."""
    gart, lib = _lib()
    for rows, cols in ((0, 8), (4, 0), (0, 0)):
        m = ctypes.byref(_m(gart, 0, rows, cols))
        assert lib.gart_layer_norm(m, None, None, 1e-5, 0, m, None) == 0
        assert lib.gart_layer_norm_backward_scratch_bytes(rows, cols, 0) == 0
    m = ctypes.byref(_m(gart, 0, 4, 0))
    assert lib.gart_layer_norm_backward(m, m, None, 1e-5, 0, m, None, None, None, 0, None) == 0
    m = ctypes.byref(_m(gart, 0, 0, 8))
    assert lib.gart_layer_norm_backward(m, m, None, 1e-5, 0, m, None, None, None, 0, None) == 0


def test_scratch_sizes():
    _, lib = _lib()
    size = lib.gart_layer_norm_backward_scratch_bytes
    assert size(-1, 8, 0) == 0 and size(8, 1 << 31, 0) == 0 and size(8, 8, 5) == 0
    for rows, cols in ((1, 1), (1 << 20, 1), (1, 1 << 20), (1_000_000, 64), (8191, 16384)):
        for t in range(3):
            assert 0 <= size(rows, cols, t) <= rows * cols * 8 + (1 << 20) + 64 * cols * 1024


@pytest.mark.parametrize("rows,cols", [(3, 2), (5, 7), (4, 33)])
def test_reference_gradient_against_differences(rows, cols):
    rng = np.random.default_rng(rows)
    x, dl = rng.standard_normal((rows, cols)) + 0.5, rng.standard_normal((rows, cols))
    gain, bias = rng.standard_normal(cols), rng.standard_normal(cols)
    grads = ref.norm_grads(x, dl, gain, 1e-2)
    for q, g in enumerate(grads):
        base = [x, gain, bias]
        v, loss = rng.standard_normal(base[q].shape), []
        for s in (1e-5, -1e-5):
            p = list(base)
            p[q] = p[q] + s * v
            loss.append((dl * ref.norm(*p, 1e-2)).sum())
        assert abs((g * v).sum() - (loss[0] - loss[1]) / 2e-5) <= 1e-6 * np.abs(dl).sum()
