"""Sizes that the learned blocks refuse as UNSUPPORTED, as the header gives them, before the device is touched."""
import ctypes

import pytest

INVALID, UNSUPPORTED = -1, -4
F32, BF16, NONE = 0, 1, 0


def _m(address, rows, cols, stride=None):
    from paper_2608_17298_amd import gart
    return ctypes.byref(gart.gart_matrix(address << 44, rows, cols, cols if stride is None else stride))


@pytest.mark.parametrize("n,dim,dtype,taken", [
    ((1 << 30) - 64, 513, F32, True), (1 << 30, 513, F32, False), (1 << 30, 512, F32, True),
    (1 << 30, 1025, BF16, False), (1 << 30, 1024, BF16, True), ((1 << 31) - 1, 1 << 23, BF16, False),
    (10, (1 << 23) + 1, F32, False), (10, 1 << 23, F32, True)])
def test_embedding_gradient_limits(n, dim, dtype, taken):
    from paper_2608_17298_amd import gart
    r = gart.lib().gart_embedding_backward(5 << 44, 0, _m(1, n, dim, 0), 1.0, dtype, _m(2, 9, dim), None, 0, None)
    assert r == (INVALID if taken else UNSUPPORTED)
    if taken:  # only the scratch is missing
        assert "scratch" in gart.lib().gart_last_error().decode()


@pytest.mark.parametrize("rows,inputs,outputs,taken", [
    (1 << 29, 1000, 64, True), ((1 << 29) + 1, 1000, 64, False), (1 << 20, 1000, 1 << 15, True),
    ((1 << 20) + 1, 1000, 1 << 15, False), (64, 1000, 1 << 24, True), (65, 1000, 1 << 29, False),
    ((1 << 31) - 1, 32, 64, True)])
@pytest.mark.parametrize("dtype", [F32, BF16])
def test_linear_limits(rows, inputs, outputs, taken, dtype):
    """The forward's; scratch that is missing or a residual on y comes after the sizes."""
    from paper_2608_17298_amd import gart
    L = gart.lib()
    x, w, y = _m(1, rows, inputs, 0), _m(2, outputs, inputs, 0), _m(3, rows, outputs)
    bad = ctypes.byref(gart.gart_matrix((3 << 44) + 4, rows, outputs, outputs))  # a residual that overlaps y
    r = L.gart_linear(x, w, None, bad, NONE, dtype, y, None, 0, None)
    assert r == (INVALID if taken else UNSUPPORTED), L.gart_last_error().decode()


@pytest.mark.parametrize("rows,inputs,outputs,taken", [
    (1 << 20, 1 << 15, 1 << 12, True), ((1 << 20) + 1, 1 << 15, 1 << 12, False), (100, 1000, 4194240, True),
    (100, 1000, 4194241, False), (100, 100_000, 400_000, False), ((1 << 31) - 1, 32, 64, True)])
@pytest.mark.parametrize("dtype", [F32, BF16])
def test_linear_gradient_limits(rows, inputs, outputs, taken, dtype):
    from paper_2608_17298_amd import gart
    L = gart.lib()
    x, w, d = _m(1, rows, inputs, 0), _m(2, outputs, inputs, 0), _m(3, rows, outputs, 0)
    need = L.gart_linear_backward_scratch_bytes(rows, inputs, outputs, dtype, NONE)
    g_x = _m(1, rows, inputs)  # begins where x does, if the scratch does not refuse the call first
    r = L.gart_linear_backward(x, w, None, NONE, d, dtype, g_x, None, None, 6 << 44, need, None)
    assert r == (INVALID if taken else UNSUPPORTED), L.gart_last_error().decode()
    assert taken or need == 0
