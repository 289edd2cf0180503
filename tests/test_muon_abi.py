"""CPU checks of the orthogonalised steps' C ABI: invalid arguments are refused before the device is touched, sizes of
scratch, the structs' layouts; and of the reference: singular values move as the polynomial says."""
import ctypes
import os
import subprocess

import numpy as np
import pytest

import muon_ref as ref

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
INVALID, MB, NAN = -1, 1 << 20, float("nan")


def _lib():
    from paper_2608_17298_amd import gart
    return gart, gart.lib()


def _m(gart, addr, rows, cols, stride=None):
    return ctypes.byref(gart.gart_matrix(addr, rows, cols, cols if stride is None else stride))


def _how(gart, **kw):
    return gart.gart_newton_schulz(*{**dict(a=3.4445, b=-4.775, c=2.0315, eps=1e-7, steps=5), **kw}.values())


HOW_BAD = dict(
    steps=("steps", dict(steps=0)), too_many=("steps", dict(steps=65)), negative=("steps", dict(steps=-1)),
    eps=("eps", dict(eps=-1.0)), eps_nan=("eps", dict(eps=NAN)), a=("coefficients", dict(a=NAN)),
    b=("coefficients", dict(b=float("inf"))), c=("coefficients", dict(c=-float("inf"))),
    grows=("1024", dict(a=10.0, b=0.0, c=0.0)), explodes=("1024", dict(a=2.0, b=3.0, c=1.0)),
    huge=("1024", dict(a=1.0, b=1e30, c=-1e30, steps=1)))


@pytest.mark.parametrize("name", sorted(HOW_BAD))
def test_iterations_refused(name):
    gart, lib = _lib()
    word, change = HOW_BAD[name]
    how = _how(gart, **change)
    need = lib.gart_orthogonalize_scratch_bytes(4, 8, 0)
    r = lib.gart_orthogonalize(_m(gart, MB, 4, 8), ctypes.byref(how), 0, _m(gart, 2 * MB, 4, 8), 8 * MB, need, None)
    assert r == INVALID and word in lib.gart_last_error().decode()
    h = gart.gart_muon(0.02, 0.95, 0.0, 1.0, 1, how)
    r = lib.gart_muon_step(_m(gart, MB, 4, 8), _m(gart, 2 * MB, 4, 8), _m(gart, 3 * MB, 4, 8), ctypes.byref(h), 0,
                           8 * MB, need, None)
    assert r == INVALID and word in lib.gart_last_error().decode()


CALL_BAD = dict(
    x_null=("x data", dict(x=(0, 4, 8))), size=("differ in size", dict(y=(2 * MB, 8, 4))),
    x_stride=("row stride", dict(x=(MB, 4, 8, 7))), y_stride0=("row stride", dict(y=(2 * MB, 4, 8, 0))),
    unaligned=("aligned", dict(x=(MB + 2, 4, 8))), overlaps=("overlaps x", dict(y=(MB + 16, 4, 8))),
    dtype=("dtype", dict(dtype=3)), no_scratch=("scratch is NULL", dict(scratch=None)),
    short=("scratch_bytes", dict(short=1)), scratch_odd=("16-byte", dict(scratch=8 * MB + 8)),
    scratch_on_x=("scratch overlaps", dict(scratch=MB + 16)), scratch_on_y=("scratch overlaps", dict(scratch=2 * MB + 16)))


@pytest.mark.parametrize("name", sorted(CALL_BAD))
def test_orthogonalize_refusals(name):
    gart, lib = _lib()
    a = dict(x=(MB, 4, 8), y=(2 * MB, 4, 8), dtype=0, scratch=8 * MB, short=0)
    word, change = CALL_BAD[name]
    a.update(change)
    need = lib.gart_orthogonalize_scratch_bytes(4, 8, 0)
    r = lib.gart_orthogonalize(_m(gart, *a["x"]), ctypes.byref(_how(gart)), a["dtype"], _m(gart, *a["y"]),
                               a["scratch"], need - a["short"], None)
    assert r == INVALID and word in lib.gart_last_error().decode(), lib.gart_last_error()


STEP_BAD = dict(
    grad_size=("grad and param", dict(grad=(2 * MB, 4, 7))), m_size=("m and param", dict(m=(3 * MB, 5, 8))),
    m_unaligned=("aligned", dict(m=(3 * MB + 2, 4, 8), dtype=1)), m_null=("m data", dict(m=(0, 4, 8))),
    param_repeated=("row stride", dict(param=(MB, 4, 8, 0))), m_repeated=("row stride", dict(m=(3 * MB, 4, 8, 0))),
    grad_is_param=("overlap", dict(grad=(MB, 4, 8))), m_is_param=("overlap", dict(m=(MB, 4, 8))),
    m_is_grad=("overlap", dict(m=(2 * MB, 4, 8))), scratch_on_m=("overlap", dict(scratch=3 * MB + 16)),
    lr=("lr", dict(lr=0.0)), lr_nan=("lr", dict(lr=NAN)), momentum=("momentum", dict(momentum=1.0)),
    momentum_low=("momentum", dict(momentum=-0.1)), decay=("weight_decay", dict(decay=-1.0)),
    scale=("scale", dict(scale=0.0)), scale_inf=("scale", dict(scale=float("inf"))),
    short=("scratch_bytes", dict(short=1)), dtype=("dtype", dict(dtype=-1)))


@pytest.mark.parametrize("name", sorted(STEP_BAD))
def test_muon_refusals(name):
    gart, lib = _lib()
    a = dict(param=(MB, 4, 8), grad=(2 * MB, 4, 8), m=(3 * MB, 4, 8), lr=0.02, momentum=0.95, decay=0.01, scale=1.0,
             dtype=0, scratch=8 * MB, short=0)
    word, change = STEP_BAD[name]
    a.update(change)
    h = gart.gart_muon(a["lr"], a["momentum"], a["decay"], a["scale"], 1, _how(gart))
    need = lib.gart_muon_scratch_bytes(4, 8, 0)
    r = lib.gart_muon_step(_m(gart, *a["param"]), _m(gart, *a["grad"]), _m(gart, *a["m"]), ctypes.byref(h), a["dtype"],
                           a["scratch"], need - a["short"], None)
    assert r == INVALID and word in lib.gart_last_error().decode(), lib.gart_last_error()


def test_null_structs_refused():
    gart, lib = _lib()
    x, y = _m(gart, MB, 4, 8), _m(gart, 2 * MB, 4, 8)
    assert lib.gart_orthogonalize(x, None, 0, y, 8 * MB, MB, None) == INVALID
    assert lib.gart_muon_step(x, y, _m(gart, 3 * MB, 4, 8), None, 0, 8 * MB, MB, None) == INVALID
    h = gart.gart_muon(0.02, 0.95, 0.0, 1.0, 1, _how(gart))
    for p in ((None, y, x), (x, None, y), (x, y, None)):
        assert lib.gart_muon_step(*p, ctypes.byref(h), 0, 8 * MB, MB, None) == INVALID


def test_empty_calls_and_scratch():
    gart, lib = _lib()
    how, size = _how(gart), lib.gart_orthogonalize_scratch_bytes
    h = gart.gart_muon(0.02, 0.95, 0.0, 1.0, 1, how)
    for rows, cols in ((0, 8), (4, 0), (0, 0)):
        e = _m(gart, 0, rows, cols)
        assert size(rows, cols, 0) == 0
        assert lib.gart_orthogonalize(e, ctypes.byref(how), 0, e, None, 0, None) == 0
        assert lib.gart_muon_step(e, e, e, ctypes.byref(h), 0, None, 0, None) == 0
    assert size(-1, 8, 0) == 0 and size(8, 1 << 31, 0) == 0 and size(8, 8, 3) == 0
    for rows, cols in ((1, 1), (48, 64), (1024, 4096), (4096, 1024), (1, 100000)):
        assert 0 < size(rows, cols, 1) == lib.gart_muon_scratch_bytes(rows, cols, 1)
    # a large weight's scratch stays within a few times its size in float32
    assert size(1024, 4096, 0) <= 5 * 4 * 1024 * 4096
    x = _m(gart, MB, 1 << 30, 1 << 30)
    assert lib.gart_orthogonalize(x, ctypes.byref(how), 0, x, 8 * MB, MB, None) == -4  # beyond a launch


def test_struct_layouts(tmp_path):
    """gart_newton_schulz and gart_muon as the C compiler lays them out."""
    from paper_2608_17298_amd import gart
    src = tmp_path / "s.c"
    rows = [(t, f) for t in ("gart_newton_schulz", "gart_muon") for f, _ in getattr(gart, t)._fields_]
    prints = "".join(f'printf("%zu\\n", offsetof({t}, {f}));' for t, f in rows)
    src.write_text('#include <stddef.h>\n#include <stdio.h>\n#include "gart.h"\nint main(void){printf("%zu %zu\\n", '
                   "sizeof(gart_newton_schulz), sizeof(gart_muon));" + prints + "return 0;}")
    subprocess.run(["gcc", "-I", os.path.join(ROOT, "include"), str(src), "-o", str(tmp_path / "s")], check=True)
    out = subprocess.run([str(tmp_path / "s")], capture_output=True, text=True, check=True).stdout.split()
    assert [int(v) for v in out[:2]] == [ctypes.sizeof(gart.gart_newton_schulz), ctypes.sizeof(gart.gart_muon)]
    assert [int(v) for v in out[2:]] == [getattr(getattr(gart, t), f).offset for t, f in rows]


@pytest.mark.parametrize("rows,cols", [(1, 5), (6, 6), (7, 20), (20, 7)])
def test_reference_moves_singular_values(rows, cols):
    rng = np.random.default_rng(rows)
    x = rng.standard_normal((rows, cols))
    u, s, v = np.linalg.svd(x, full_matrices=False)
    want = (u * ref.singular_values(s / (np.sqrt((s ** 2).sum()) + 1e-7))) @ v
    assert np.abs(ref.orthogonalize(x) - want).max() < 1e-12


@pytest.mark.parametrize("start", [1.0, 0.05, 1e-6, 1e-23])
def test_scales_cover_what_steps_reach(tmp_path, start):
    """The scales' bounds against the polynomials on a fine grid of singular values in [0, start]: every X, A and P stays
    below 2^14 of its scale's inverse, and no scale is smaller than a sixteenth of what would fit."""
    sets = [(3.4445, -4.775, 2.0315), (1.5, -0.5, 0.0), (1.875, -1.25, 0.375), (2.0, -1.5, 0.5), (-3.0, 4.0, -1.5),
            (0.5, 0.0, 0.0), (0.8, 0.0, 0.2), (0.0, 0.0, 0.0), (3.0, -3.2, 1.2)]
    src = tmp_path / "s.cpp"
    src.write_text('#include <cstdio>\n#include "orthogonalize.h"\nint main(int, char** v){ double a, b, c, z; '
                   "for (;std::scanf(\"%lf %lf %lf %lf\", &a, &b, &c, &z) == 4;) { "
                   "for (int k = 0; k < 6; ++k) { gart::StepScales s; z = gart::step_scales(a, b, c, z, &s); "
                   "std::printf(\" %.17g %.17g %.17g\", s.x, s.a, s.p); } std::printf(\"\\n\"); } }")
    exe = str(tmp_path / "s")
    subprocess.run(["g++", "-std=c++17", "-O1", "-I", os.path.join(ROOT, "paper_2608_17298_amd", "csrc"), str(src),
                    "-o", exe], check=True)
    text = "\n".join(" ".join(repr(v) for v in (*q, start)) for q in sets)
    lines = subprocess.run([exe], input=text, capture_output=True, text=True, check=True).stdout.strip().split("\n")
    for (a, b, c), line in zip(sets, lines):
        f = [float(v) for v in line.split()]
        s = np.linspace(0.0, start, 200001)
        bound = start
        for k in range(6):
            x, qa, qp = f[3 * k:3 + 3 * k]
            t = s * s
            grid = np.linspace(0.0, bound, 200001)  # the interval that the bounds take s to fill
            for value, reach, scale, most in ((s, grid, x, 120), (t, grid ** 2, qa, 60),
                                              (b * t + c * t * t, b * grid ** 2 + c * grid ** 4, qp, 60)):
                assert np.abs(value).max() * scale <= 2.0 ** 14
                top = np.abs(reach).max()
                assert top == 0 or scale == 2.0 ** most or top * scale >= 2.0 ** 10
            s = a * s + b * s ** 3 + c * s ** 5
            bound = np.abs(a * grid + b * grid ** 3 + c * grid ** 5).max()
