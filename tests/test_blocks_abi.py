"""CPU checks of the learned blocks' C ABI: invalid arguments are refused before the device is touched, sizes of
scratch, the layout of gart_matrix, and the reference forms themselves (generator, gradients by differences)."""
import ctypes
import os
import subprocess

import numpy as np
import pytest

import blocks_ref as ref

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
INVALID = -1


def _m(gart, addr, rows, cols, stride=None):
    return gart.gart_matrix(addr, rows, cols, cols if stride is None else stride)


def _err(lib):
    return lib.gart_last_error().decode()


LINEAR_BAD = dict(
    x_null=("x data", dict(x=(0, 4, 8))), stride=("row stride", dict(x=(1 << 20, 4, 8, 7))),
    negative=("-1", dict(x=(1 << 20, -1, 8))), k=("columns", dict(w=(2 << 20, 6, 9))),
    y_size=("y is", dict(y=(3 << 20, 4, 7))), y_rows=("y is", dict(y=(3 << 20, 5, 6))),
    y_stride0=("row stride", dict(y=(3 << 20, 4, 6, 0))), unaligned=("aligned", dict(x=((1 << 20) + 2, 4, 8))),
    y_is_x=("overlaps", dict(y=((1 << 20) + 16, 4, 6))), y_is_w=("overlaps", dict(y=((2 << 20) + 16, 4, 6))),
    residual_size=("residual", dict(residual=(4 << 20, 4, 5))),
    residual_overlap=("residual", dict(residual=((3 << 20) + 4, 4, 6))),
    act=("activation", dict(act=4)), dtype=("dtype", dict(dtype=3)), bias=("bias", dict(bias=(5 << 20) + 1)),
    too_many=("x is", dict(x=(1 << 20, 1 << 31, 8))))


@pytest.mark.parametrize("name", sorted(LINEAR_BAD))
def test_linear_refusals(name):
    from paper_2608_17298_amd import gart
    lib = gart.lib()
    a = dict(x=(1 << 20, 4, 8), w=(2 << 20, 6, 8), y=(3 << 20, 4, 6), residual=None, bias=None, act=0, dtype=0)
    word, change = LINEAR_BAD[name]
    a.update(change)
    m = {k: ctypes.byref(_m(gart, *a[k])) if a[k] else None for k in ("x", "w", "y", "residual")}
    r = lib.gart_linear(m["x"], m["w"], a["bias"], m["residual"], a["act"], a["dtype"], m["y"], None, 0, None)
    assert r == INVALID and word in _err(lib), _err(lib)


def test_null_matrices_refused():
    from paper_2608_17298_amd import gart
    lib = gart.lib()
    x = ctypes.byref(_m(gart, 1 << 20, 4, 8))
    assert lib.gart_linear(None, x, None, None, 0, 0, x, None, 0, None) == INVALID
    assert lib.gart_linear_backward(x, None, None, 0, x, 0, None, None, None, None, 0, None) == INVALID
    assert lib.gart_embedding(x, None, 0, 1.0, 0, None, None) == INVALID
    assert lib.gart_embedding(x, None, 0, 1.0, 0, ctypes.byref(_m(gart, 2 << 20, 3, 8)), None) == INVALID
    assert "ids" in _err(lib)
    assert lib.gart_embedding_backward(None, 0, x, 1.0, 0, None, None, 0, None) == INVALID
    assert lib.gart_dropout(x, None, 0.5, 0, 0, 0, None, None) == INVALID


@pytest.mark.parametrize("p", [-0.1, 1.01, float("nan")])
def test_dropout_rate_refused(p):
    from paper_2608_17298_amd import gart
    lib = gart.lib()
    x = ctypes.byref(_m(gart, 1 << 20, 4, 8))
    assert lib.gart_dropout(x, None, p, 0, 0, 0, x, None) == INVALID and "p must" in _err(lib)


def test_gradient_overlaps_refused():
    from paper_2608_17298_amd import gart
    lib = gart.lib()
    x, w, d = _m(gart, 1 << 20, 4, 8), _m(gart, 2 << 20, 6, 8), _m(gart, 3 << 20, 4, 6)
    need = lib.gart_linear_backward_scratch_bytes(4, 8, 6, 0, 0)
    for gx, gw, gb in [(x, None, None), (None, w, None), (_m(gart, 4 << 20, 4, 8), _m(gart, (4 << 20) + 4, 6, 8), None),
                       (None, None, 3 << 20), (_m(gart, 4 << 20, 4, 8), None, (4 << 20) + 8)]:
        q = [ctypes.byref(t) if t is not None else None for t in (x, w, d, gx, gw)]
        r = lib.gart_linear_backward(q[0], q[1], None, 0, q[2], 0, q[3], q[4], gb, 8 << 20, need, None)
        assert r == INVALID and "overlap" in _err(lib)


def test_scratch_refused():
    from paper_2608_17298_amd import gart
    lib = gart.lib()
    d, g = ctypes.byref(_m(gart, 1 << 20, 100, 8)), ctypes.byref(_m(gart, 2 << 20, 9, 8))
    need = lib.gart_embedding_scratch_bytes(100, 9, 8)
    assert need > 0
    for p, n in [(None, need), (3 << 20, need - 1), ((3 << 20) + 8, need)]:
        assert lib.gart_embedding_backward(4 << 20, 0, d, 1.0, 0, g, p, n, None) == INVALID and "scratch" in _err(lib)
    x, w, y = (ctypes.byref(_m(gart, a << 20, r, c)) for a, r, c in ((1, 300, 8), (2, 6, 8), (3, 300, 6)))
    need = lib.gart_linear_backward_scratch_bytes(300, 8, 6, 0, 2)
    for p, n in [(None, need), (8 << 20, need - 1)]:
        r = lib.gart_linear_backward(x, w, None, 2, y, 0, None, ctypes.byref(_m(gart, 5 << 20, 6, 8)), None, p, n, None)
        assert r == INVALID and "scratch" in _err(lib)


def test_scratch_overlaps_refused():
    """Scratch on an input or an output: refused, whichever it is."""
    from paper_2608_17298_amd import gart
    lib = gart.lib()
    m = lambda mb, r, c: ctypes.byref(_m(gart, mb << 20, r, c))  # noqa: E731
    need = lib.gart_embedding_scratch_bytes(100, 9, 8)
    for mb in (1, 2, 4):
        r = lib.gart_embedding_backward(4 << 20, 0, m(1, 100, 8), 1.0, 0, m(2, 9, 8), (mb << 20) + 16, need, None)
        assert r == INVALID and "scratch overlaps" in _err(lib)
    need = lib.gart_linear_scratch_bytes(300, 2000, 200, 0)
    assert 0 < need < 16 << 20
    for mb in (32, 64, 96, 128, 160):
        r = lib.gart_linear(m(32, 300, 2000), m(64, 200, 2000), 96 << 20, m(128, 300, 200), 0, 0, m(160, 300, 200),
                            (mb << 20) + 16, need, None)
        assert r == INVALID and "scratch overlaps" in _err(lib)
    need = lib.gart_linear_backward_scratch_bytes(300, 8, 6, 0, 2)
    assert 0 < need < 16 << 20
    for mb in range(32, 32 * 8, 32):
        r = lib.gart_linear_backward(m(32, 300, 8), m(64, 6, 8), 96 << 20, 2, m(128, 300, 6), 0, m(160, 300, 8),
                                     m(192, 6, 8), 224 << 20, (mb << 20) + 16, need, None)
        assert r == INVALID and "scratch overlaps" in _err(lib)


def test_scratch_sizes():
    from paper_2608_17298_amd import gart
    lib = gart.lib()
    for empty in ((0, 5, 5), (5, 0, 5), (5, 5, 0), (0, 0, 0)):
        assert lib.gart_embedding_scratch_bytes(*empty) == 0
        lib.gart_linear_scratch_bytes(*empty, 0)
        lib.gart_linear_backward_scratch_bytes(*empty, 1, 2)
    assert lib.gart_embedding_scratch_bytes(0, 5, 5) == 0 and lib.gart_embedding_scratch_bytes(-1, 5, 5) == 0
    assert lib.gart_linear_backward_scratch_bytes(-1, 5, 5, 0, 0) == 0
    assert lib.gart_linear_backward_scratch_bytes(10, 5, 5, 7, 0) == 0
    assert lib.gart_linear_backward_scratch_bytes(10, 5, 5, 0, 9) == 0
    a = [lib.gart_embedding_scratch_bytes(n, 100, 64) for n in (100, 1000, 10000)]
    assert 0 < a[0] < a[1] < a[2]
    # gradients of a million rows keep within a few times the inputs
    need = lib.gart_linear_backward_scratch_bytes(1_000_000, 64, 128, 1, 2)
    assert need <= 1_000_000 * 128 * 2 * 2


def test_interleaved_columns_are_no_overlap():
    """x and y as columns of one buffer: accepted up to the launch (no rows, so none follows)."""
    from paper_2608_17298_amd import gart
    lib = gart.lib()
    x, w, y = _m(gart, 1 << 20, 4, 8, 20), _m(gart, 2 << 20, 6, 8), _m(gart, (1 << 20) + 36, 4, 6, 20)
    inside = _m(gart, (1 << 20) + 28, 4, 6, 20)
    r = lib.gart_linear(ctypes.byref(x), ctypes.byref(w), None, None, 0, 0, ctypes.byref(inside), None, 0, None)
    assert r == INVALID and "overlaps" in _err(lib)  # begins inside x's eight columns
    r = lib.gart_linear(ctypes.byref(x), ctypes.byref(w), None, ctypes.byref(_m(gart, 5 << 20, 4, 5)), 0, 0,
                        ctypes.byref(y), None, 0, None)
    assert r == INVALID and "overlaps" not in _err(lib)  # beside them: only the residual's size is wrong


def test_empty_calls_need_nothing():
    from paper_2608_17298_amd import gart
    lib = gart.lib()
    e = lambda r, c: ctypes.byref(_m(gart, 0, r, c))  # noqa: E731
    w = ctypes.byref(_m(gart, 1 << 20, 6, 8))
    assert lib.gart_linear(e(0, 8), w, None, None, 1, 1, e(0, 6), None, 0, None) == 0
    assert lib.gart_embedding(ctypes.byref(_m(gart, 1 << 20, 6, 8)), None, 1, 1.0, 0, e(0, 8), None) == 0
    assert lib.gart_dropout(e(0, 3), None, 0.5, 0, 0, 2, e(0, 3), None) == 0
    assert lib.gart_embedding_backward(None, 0, e(0, 0), 1.0, 0, e(5, 0), None, 0, None) == 0


def test_matrix_struct_matches_header(tmp_path):
    from paper_2608_17298_amd import gart
    src = tmp_path / "m.c"
    fields = [f[0] for f in gart.gart_matrix._fields_]
    src.write_text('#include <stdio.h>\n#include <stddef.h>\n#include "gart.h"\nint main(void) {\n'
                   + "".join(f'  printf("%zu ", offsetof(gart_matrix, {f}));\n' for f in fields)
                   + '  printf("%zu %d %d %d %d\\n", sizeof(gart_matrix), GART_DTYPE_BF16, GART_DTYPE_F16,'
                     ' GART_ACT_SILU, GART_ACT_GELU);\n  return 0;\n}\n')
    exe = tmp_path / "m"
    subprocess.run(["gcc", "-std=c11", "-I", os.path.join(ROOT, "include"), str(src), "-o", str(exe)], check=True)
    got = [int(v) for v in subprocess.run([str(exe)], check=True, capture_output=True, text=True).stdout.split()]
    want = [getattr(gart.gart_matrix, f).offset for f in fields]
    assert got == want + [ctypes.sizeof(gart.gart_matrix), gart.DTYPE_BF16, gart.DTYPE_F16, gart.ACT_SILU,
                          gart.ACT_GELU]


def test_generator_known_answers():
    """Vectors published with the generator: all-zero and all-one counters and keys."""
    assert ref.philox(0, 0, 0) == [0x6627E8D5, 0xE169C58D, 0xBC57AC4C, 0x9B00DBD8]
    ones = (1 << 64) - 1
    assert ref.philox(ones, ones, ones) == [0x408F276D, 0x41C83B0E, 0xA20BC7C6, 0x6D5451FD]


@pytest.mark.parametrize("name", ["none", "silu", "gelu"])
def test_reference_gradients_by_differences(name):
    rng = np.random.default_rng(0)
    z = np.linspace(-9, 9, 181)
    h = 1e-5
    d = (ref.act(z + h, name) - ref.act(z - h, name)) / (2 * h)
    assert np.abs(d - ref.act_grad(z, name)).max() <= 1e-9
    x, w, b, dl = (rng.standard_normal(s) for s in ((5, 3), (4, 3), 4, (5, 4)))
    gx, gw, gb = ref.linear_grads(x, w, b, dl, name)
    f = lambda x, w, b: (dl * ref.linear(x, w, b, None, name)).sum()  # noqa: E731
    for q, g in enumerate((gx, gw, gb)):
        v = rng.standard_normal(g.shape)
        p, m = [x, w, b], [x, w, b]
        p[q], m[q] = p[q] + h * v, m[q] - h * v
        assert abs((f(*p) - f(*m)) / (2 * h) - (g * v).sum()) <= 1e-7
