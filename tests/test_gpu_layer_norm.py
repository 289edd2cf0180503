"""The layer norm and its gradient on the GPU against plain 64-bit forms: sizes from nothing and one element up, odd and
strided rows, rows longer than registers hold, every type, constant rows, non-finite values, offsets beyond 32 bits,
other streams, graphs, repeatability.  Gradients also against central differences."""
import numpy as np
import pytest

import blocks_ref
import layer_norm_ref as ref
from test_gpu_blocks import GUARD, TYPES, _Out, _inside, _integers, _mat, _rounded, _scratch, _torch, _vec, _within

pytestmark = pytest.mark.gpu

EPS = 1e-5
EPS32 = float(np.float32(EPS))
SIZES = [(1, 1), (1, 2), (7, 1), (300, 3), (5, 4), (9, 5), (1000, 7), (3, 8), (64, 9), (129, 16), (33, 17), (100, 48),
         (1, 1024), (501, 32), (2000, 33), (70, 64), (31, 100), (40, 127), (20, 129), (65, 255), (17, 260), (13, 511),
         (9, 513), (7, 1023), (6, 1025), (5, 2047), (5, 2050), (3, 4095), (3, 4104), (3, 8191), (2, 8200), (2, 16383),
         (2, 16392), (1, 40001), (2, 70000), (5000, 12), (9001, 5), (4097, 64)]
EMPTY = [(0, 5), (5, 0), (0, 0)]


def _rows(rng, rows, cols, dtype, pad=0):
    """Rows of different sizes, off their middle."""
    import torch
    v = rng.standard_normal((rows, cols + pad)) * np.exp(0.5 * rng.standard_normal((rows, 1))) \
        + rng.standard_normal((rows, 1))
    t = torch.from_numpy(v).to(_torch(dtype)).cuda()[:, :cols]
    return t, t.cpu().double().numpy()


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("rows,cols", SIZES + EMPTY)
@pytest.mark.parametrize("gain,bias,pad", [(True, True, 0), (False, True, 3), (True, False, 8), (False, False, 1)])
def test_layer_norm(rows, cols, dtype, gain, bias, pad):
    from paper_2608_17298_amd import gart
    rng = np.random.default_rng(rows + 10 * cols)
    x, x64 = _rows(rng, rows, cols, dtype, pad)
    g, g64 = _vec(rng, cols, dtype) if gain else (None, None)
    b, b64 = _vec(rng, cols, dtype) if bias else (None, None)
    y = _Out(rows, cols, dtype, 2 * pad)
    gart.gart_layer_norm(x, y.t, g, b, EPS)
    if rows * cols == 0:
        assert y.value().size == 0
        return
    _within(y.value(), ref.norm(x64, g64, b64, EPS32), ref.norm_tolerance(x64, g64, b64, EPS32, dtype))


def _grads(x, dl, gain, dtype, pad=0, eps=EPS):
    from paper_2608_17298_amd import gart
    rows, cols = x.shape
    gx, gg, gb = _Out(rows, cols, dtype, pad), _Out(1, cols, dtype, 0), _Out(1, cols, dtype, 0)
    gart.gart_layer_norm_backward(x, dl, gx.t, gg.t.reshape(-1), gb.t.reshape(-1), gain, eps, _scratch(
        gart.gart_layer_norm_backward_scratch_bytes(rows, cols, _torch(dtype))))
    return gx.value(), gg.value()[0], gb.value()[0]


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("rows,cols", SIZES + EMPTY)
@pytest.mark.parametrize("gain,pad", [(True, 0), (False, 3), (True, 8)])
def test_layer_norm_backward(rows, cols, dtype, gain, pad):
    rng = np.random.default_rng(3 * rows + cols)
    x, x64 = _rows(rng, rows, cols, dtype, pad)
    dl, d64 = _mat(rng, rows, cols, dtype, 2 * pad)
    g, g64 = _vec(rng, cols, dtype) if gain else (None, None)
    got = [_grads(x, dl, g, dtype, pad) for _ in range(2)]
    if rows * cols == 0:
        assert all((v == 0).all() for v in got[0][1:])  # sums of nothing
        return
    want, tol = ref.norm_grads(x64, d64, g64, EPS32), ref.norm_grads_tolerance(x64, d64, g64, EPS32, dtype)
    for a, b, w, t in zip(*got, want, tol):
        assert np.array_equal(a, b)  # deterministic
        _within(a, w, t)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("rows,cols,pad", [(70001, 8, 0), (300007, 2, 0), (100000, 34, 3), (20000, 256, 0),
                                           (20001, 510, 8), (3000, 2046, 1), (1100, 3000, 3), (1000, 9000, 0), (300, 17000, 0),
                                           (129, 5000, 1), (128, 5000, 0)])
def test_column_sums_are_exact_in_whole_numbers(rows, cols, pad, dtype):
    """Rows of as many 1 as -1 with eps = 0: mean 0, variance 1 and h = x exactly, so the sums over rows are of whole
    numbers below 2^24, exact in float in any order, and rounded once: every row is in them, once."""
    rng = np.random.default_rng(rows)
    x64 = rng.permuted(np.tile(np.where(np.arange(cols) % 2, 1.0, -1.0), (rows, 1)).astype(np.float32), axis=1)
    x = _inside(x64, dtype, pad, 0.0)
    dl, d64 = _integers(rng, rows, cols, dtype, pad, 2)
    _, gg, gb = _grads(x, dl, None, dtype, pad, 0.0)
    for got, want in ((gg, (d64 * x64).sum(axis=0, dtype=np.float64)), (gb, d64.sum(axis=0))):
        assert np.abs(want).max() < 60000
        assert np.array_equal(got, _rounded(want, dtype))


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("rows,cols", [(400000, 9), (200000, 40), (30000, 300), (4000, 5000)])
def test_many_rows(rows, cols, dtype):
    """More rows than one turn of the grid has; the last ones, and others throughout, against the 64-bit form."""
    import torch
    from paper_2608_17298_amd import gart
    rng = np.random.default_rng(cols)
    x, x64 = _rows(rng, rows, cols, dtype)
    dl, d64 = _mat(rng, rows, cols, dtype)
    g, g64 = _vec(rng, cols, dtype)
    y = torch.empty_like(x)
    gart.gart_layer_norm(x, y, g, None, EPS)
    pick = np.concatenate([np.arange(0, rows, 997), np.arange(rows - 50, rows)])
    _within(y.cpu().double().numpy()[pick], ref.norm(x64[pick], g64, None, EPS32),
            ref.norm_tolerance(x64[pick], g64, None, EPS32, dtype))
    gx, gg, gb = _grads(x, dl, g, dtype)
    want, tol = ref.norm_grads(x64[pick], d64[pick], g64, EPS32), ref.norm_grads_tolerance(x64[pick], d64[pick], g64,
                                                                                         EPS32, dtype)
    _within(gx[pick], want[0], tol[0])
    want, tol = ref.norm_grads(x64, d64, g64, EPS32), ref.norm_grads_tolerance(x64, d64, g64, EPS32, dtype)
    _within(gg, want[1], tol[1])
    _within(gb, want[2], tol[2])


@pytest.mark.parametrize("want_x,want_gain,want_bias", [(1, 0, 0), (0, 1, 0), (0, 0, 1), (1, 0, 1), (0, 0, 0)])
@pytest.mark.parametrize("rows,cols", [(300, 40), (20, 3000), (3, 20000)])
def test_some_outputs(want_x, want_gain, want_bias, rows, cols):
    """Gradients that are not asked for change nothing in the others."""
    import torch
    from paper_2608_17298_amd import gart
    rng = np.random.default_rng(5)
    (x, _), (dl, _), (g, _) = _rows(rng, rows, cols, "f32"), _mat(rng, rows, cols, "f32"), _vec(rng, cols, "f32")
    scratch = _scratch(gart.gart_layer_norm_backward_scratch_bytes(rows, cols))
    full = [torch.empty_like(x), torch.empty_like(g), torch.empty_like(g)]
    gart.gart_layer_norm_backward(x, dl, *full, g, EPS, scratch)
    some = [torch.empty_like(t) if f else None for t, f in zip(full, (want_x, want_gain, want_bias))]
    gart.gart_layer_norm_backward(x, dl, *some, g, EPS, scratch)
    for a, b in zip(full, some):
        assert b is None or torch.equal(a, b)


@pytest.mark.parametrize("rows,cols", [(20, 6), (9, 300), (3, 2500)])
def test_backward_against_differences(rows, cols):
    """d(sum dl y) along random directions of x, gain and bias, by central differences in 64 bits."""
    rng = np.random.default_rng(11)
    (x, x64), (dl, d64), (g, g64) = _rows(rng, rows, cols, "f32"), _mat(rng, rows, cols, "f32"), _vec(rng, cols, "f32")
    got, tol = _grads(x, dl, g, "f32"), ref.norm_grads_tolerance(x64, d64, g64, EPS32, "f32")
    base, h = [x64, g64, np.zeros(cols)], 1e-5
    for q in range(3):
        v = rng.standard_normal(base[q].shape)
        loss = []
        for sign in (1.0, -1.0):
            p = list(base)
            p[q] = p[q] + sign * h * v
            loss.append((d64 * ref.norm(*p, EPS32)).sum())
        slope = (loss[0] - loss[1]) / (2 * h)
        # the differences' own error: a third derivative is at most 15 rstd^3 |v|^3 of each term; 64-bit rounding over 2h
        rstd = 1.0 / x64.std(axis=1).min()
        own = (0 if q else 15 * (h * rstd) ** 2 * rstd * (np.abs(d64 * g64) * np.abs(v).max() ** 3).sum()) \
            + 1e-14 * np.abs(d64).sum() * 10 / h
        assert abs((got[q] * v).sum() - slope) <= (tol[q] * np.abs(v)).sum() + own


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("cols", [1, 6, 64, 999, 5000, 20000])
def test_constant_rows(cols, dtype):
    """A row of one value (all of a column's rows, with one column): h is 0, y is the bias, the gradients are finite."""
    import torch
    from paper_2608_17298_amd import gart
    t = _torch(dtype)
    x = torch.full((3, cols), 0.5, dtype=t, device="cuda")  # sums of halves are exact
    b = torch.arange(cols, device="cuda").remainder(7).to(t)
    y = torch.empty_like(x)
    gart.gart_layer_norm(x, y, None, b, EPS)
    assert torch.equal(y, b.expand(3, cols))
    dl = torch.ones_like(x)
    gx, gg, gb = _grads(x, dl, None, dtype)
    assert (gx == 0).all() and (gg == 0).all() and (gb == 3).all()


@pytest.mark.parametrize("cols", [5, 64, 1000, 9000])
def test_mean_far_from_zero(cols):
    """Whole numbers around 1024: their sum is exact in float, so the mean is off by its division alone, and each
    difference by that and its own rounding.  A difference of squares would lose the variance."""
    import torch
    from paper_2608_17298_amd import gart
    rng = np.random.default_rng(cols)
    x64 = 1024.0 + rng.integers(-4, 5, (6, cols))
    x = torch.from_numpy(x64.astype(np.float32)).cuda()
    y = torch.empty_like(x)
    gart.gart_layer_norm(x, y, None, None, EPS)
    u, d = blocks_ref.U32, x64 - x64.mean(axis=1, keepdims=True)
    var = (d * d).mean(axis=1, keepdims=True) + EPS32
    e_d = 2 * u * 1030 + u * np.abs(d)
    # the differences' common error is at right angles to them: their squares keep its square alone
    e_var = (80 + cols / 256 + 5) * u * var + (2 * u * 1030) ** 2 + 2 * u * (d * d).mean(axis=1, keepdims=True)
    tol = 1.1 * (e_d / np.sqrt(var) + np.abs(d) / np.sqrt(var) * (0.5 * e_var / var + 10 * u))
    _within(y.cpu().double().numpy(), ref.norm(x64, None, None, EPS32), tol)


def test_small_and_large_variances():
    """Variances from subnormal floats to 1e36, with eps = 0: |y| of a row of +s and -s is 1."""
    import torch
    from paper_2608_17298_amd import gart
    s = np.array([2.0 ** -70, 2.0 ** -60, 2.0 ** -50, 1e-6, 1.0, 1e9, 1e18], dtype=np.float32)
    x = torch.from_numpy(np.stack([s, -s, s, -s], axis=1)).cuda()
    y = torch.empty_like(x)
    gart.gart_layer_norm(x, y, None, None, 0.0)
    got = np.abs(y.cpu().double().numpy())
    assert (np.abs(got[1:] - 1.0) <= 8 * blocks_ref.U32).all()
    assert (np.abs(got[0] - 1.0) <= 2.0 ** -8).all()  # 2^-140 has ten bits above the smallest subnormal


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("rows,cols,pad", [(5, 1, 3), (40, 3, 1), (40, 33, 3), (9, 1023, 1), (7, 2050, 8), (5, 9001, 3),
                                           (3, 20000, 1), (3000, 64, 8)])
def test_uses_nothing_around_its_inputs(rows, cols, pad, dtype):
    """NaN before, behind and between the rows of every input: the results are those with zeros there, bit for bit."""
    import torch
    from paper_2608_17298_amd import gart
    rng = np.random.default_rng(7 * rows + cols)
    x, dl = rng.standard_normal((rows, cols)), rng.standard_normal((rows, cols))
    g, b, t = rng.standard_normal((1, cols)), rng.standard_normal((1, cols)), _torch(dtype)
    got = []
    for around in (0.0, float("nan")):
        dx, dd = (_inside(v, dtype, pad, around) for v in (x, dl))
        dg, db = (_inside(v, dtype, 0, around).reshape(-1) for v in (g, b))
        y = torch.empty((rows, cols), dtype=t, device="cuda")
        gart.gart_layer_norm(dx, y, dg, db, EPS)
        o = [torch.empty(q, dtype=t, device="cuda") for q in ((rows, cols), (cols,), (cols,))]
        gart.gart_layer_norm_backward(dx, dd, *o, dg, EPS, _scratch(
            gart.gart_layer_norm_backward_scratch_bytes(rows, cols, t)))
        got.append([y, *o])
    for zeros, nans in zip(*got):
        assert torch.isfinite(zeros).all() and torch.equal(zeros, nans)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("value", [float("nan"), float("inf"), -float("inf")])
@pytest.mark.parametrize("rows,cols", [(9, 3), (70, 40), (9, 1023), (5, 5000), (3, 20000)])
def test_nonfinite_stays_in_its_row(rows, cols, value, dtype):
    """One element that is no finite number: its row of y and g_x is NaN, every other row as without it."""
    import torch
    from paper_2608_17298_amd import gart
    rng = np.random.default_rng(rows)
    x, _ = _rows(rng, rows, cols, dtype)
    dl, _ = _mat(rng, rows, cols, dtype)
    y0, y1 = torch.empty_like(x), torch.empty_like(x)
    gart.gart_layer_norm(x, y0, None, None, EPS)
    g0 = _grads(x, dl, None, dtype)
    x[rows // 2, cols - 1] = value
    gart.gart_layer_norm(x, y1, None, None, EPS)
    g1 = _grads(x, dl, None, dtype)
    bad = np.arange(rows) == rows // 2
    for a, b in ((y0.cpu().double().numpy(), y1.cpu().double().numpy()), (g0[0], g1[0])):
        assert np.isnan(b[bad]).all() and np.array_equal(a[~bad], b[~bad])
    assert np.isnan(g1[1]).all() and np.array_equal(g0[2], g1[2])


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("cols", [6, 13, 50, 130, 1023, 2047, 5001, 9001])
def test_infinite_dl_is_the_same_at_both_ends_of_a_row(cols, dtype):
    """Packs overlap at a row's end: what is infinite there counts once, as at the beginning.  With dl = (inf, 1, 1 ..)
    mean(w) is infinite, so g_x is the NaN or the infinity that the formula has."""
    import torch
    rng = np.random.default_rng(cols)
    x, x64 = _rows(rng, 3, cols, dtype)
    for at in (0, cols - 1, cols - 2):
        dl = torch.ones_like(x)
        dl[1, at] = float("inf")
        gx, gg, gb = _grads(x, dl, None, dtype)
        with np.errstate(invalid="ignore"):
            want, want_gain, _ = ref.norm_grads(x64, dl.cpu().double().numpy(), None, EPS32)
        assert np.array_equal(np.isnan(gx), np.isnan(want)) and np.array_equal(np.isinf(gx), np.isinf(want))
        assert np.isinf(gb[at]) and np.isfinite(np.delete(gb, at)).all() and np.isfinite(np.delete(gg, at)).all()
        assert not np.isnan(gg[at])


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("rows,cols,pad", [(33, 5, 3), (100, 48, 0), (9, 1023, 1), (5, 5000, 8), (3, 17001, 3),
                                           (2, 70001, 0)])
def test_in_place_and_repeated_rows(rows, cols, pad, dtype):
    """y written over x; x and dl as one row repeated (stride 0)."""
    import torch
    from paper_2608_17298_amd import gart
    rng = np.random.default_rng(cols)
    x, _ = _rows(rng, rows, cols, dtype, pad)
    (g, _), (b, _) = _vec(rng, cols, dtype), _vec(rng, cols, dtype)
    y = torch.empty((rows, cols), dtype=x.dtype, device="cuda")
    gart.gart_layer_norm(x, y, g, b, EPS)
    one = x[:1].clone()
    gart.gart_layer_norm(x, x, g, b, EPS)
    assert torch.equal(x, y)
    z = torch.empty_like(y)
    gart.gart_layer_norm(one.expand(rows, cols), z, g, b, EPS)
    assert torch.equal(z, y[:1].expand(rows, cols))
    dl, _ = _mat(rng, 1, cols, dtype)
    same = _grads(one.expand(rows, cols), dl.expand(rows, cols), g, dtype)
    for p, q in zip(same, _grads(one.repeat(rows, 1), dl.repeat(rows, 1), g, dtype)):
        assert np.array_equal(p, q)


def test_rounding_of_the_elements_type():
    """16-bit results are the 64-bit ones rounded once, but for the few whose neighbourhood of a border float32 crosses."""
    import torch
    from paper_2608_17298_amd import gart
    rng = np.random.default_rng(1)
    for dtype in ("bf16", "f16"):
        x, x64 = _rows(rng, 200, 300, dtype)
        y = torch.empty_like(x)
        gart.gart_layer_norm(x, y, None, None, EPS)
        want = ref.norm(x64, None, None, EPS32)
        off = y.cpu().double().numpy() != _rounded(want, dtype)
        # a value within 80 + 80 float32 roundings of a border may go either way: 160 2^-24 / (eps / 2) of them
        assert off.mean() <= 160 * blocks_ref.U32 / blocks_ref.U[dtype] * 2


def test_offsets_beyond_32_bits():
    """Rows 2^22 elements apart, 1040 of them: element offsets pass 2^32."""
    import torch
    from paper_2608_17298_amd import gart
    rows, step, cols = 1040, 1 << 22, 24
    if torch.cuda.mem_get_info()[0] < 20 << 30:
        pytest.skip("needs 18 GB of device memory")
    rng = np.random.default_rng(3)
    buffers = [torch.empty((rows - 1) * step + cols, dtype=torch.bfloat16, device="cuda") for _ in range(2)]
    far = [b.as_strided((rows, cols), (step, 1)) for b in buffers]
    x, _ = _rows(rng, rows, cols, "bf16")
    far[0].copy_(x)
    near = torch.empty_like(x)
    gart.gart_layer_norm(x, near)
    gart.gart_layer_norm(far[0], far[1])
    assert torch.equal(far[1], near)
    s = _scratch(gart.gart_layer_norm_backward_scratch_bytes(rows, cols, torch.bfloat16))
    o = [[torch.empty_like(x), x.new_empty(cols), x.new_empty(cols)] for _ in range(2)]
    gart.gart_layer_norm_backward(x, near, *o[0], scratch=s)
    gart.gart_layer_norm_backward(far[0], far[1], *o[1], scratch=s)
    for a, b in zip(*o):
        assert torch.equal(a, b)
    far[1].fill_(0.0)
    out = x.clone()
    gart.gart_layer_norm_backward(far[0], out, far[1], scratch=s)
    gart.gart_layer_norm_backward(x, out, near, scratch=s)
    assert torch.equal(far[1], near)


def _calls(rows, cols, dtype="bf16"):
    import torch
    from paper_2608_17298_amd import gart
    rng = np.random.default_rng(4)
    x, dl, g, b = _rows(rng, rows, cols, dtype)[0], _mat(rng, rows, cols, dtype)[0], *(
        _vec(rng, cols, dtype)[0] for _ in range(2))
    y, gx, gg, gb = torch.empty_like(x), torch.empty_like(x), torch.empty_like(g), torch.empty_like(g)
    s = _scratch(gart.gart_layer_norm_backward_scratch_bytes(rows, cols, x.dtype))

    def run(stream=None):
        gart.gart_layer_norm(x, y, g, b, EPS, stream=stream)
        gart.gart_layer_norm_backward(y, dl, gx, gg, gb, g, EPS, s, stream=stream)

    return run, [y, gx, gg, gb]


@pytest.mark.parametrize("rows,cols", [(600, 40), (100, 3000), (4, 20000)])
def test_another_stream_and_graphs(rows, cols):
    """On a side stream, and captured once and replayed four times with other work between."""
    import torch
    run, outs = _calls(rows, cols)
    run()
    torch.cuda.synchronize()
    want = [t.clone() for t in outs]
    for t in outs:
        t.zero_()
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    run(side)
    side.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(outs, want))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        run()
    for _ in range(4):
        for t in outs:
            t.fill_(GUARD)
        (torch.randn((512, 512), device="cuda") * 2.0).sum().item()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(outs, want))


def test_refusals_on_tensors():
    """Tensors of the wrong kind are refused before the library is called, and nothing is written."""
    import torch
    from paper_2608_17298_amd import gart
    x, g = torch.ones((4, 8), device="cuda"), torch.ones(8, device="cuda")
    y = torch.full((4, 8), 5.0, device="cuda")
    bad = [lambda: gart.gart_layer_norm(x.cpu(), y), lambda: gart.gart_layer_norm(x, y.half()),
           lambda: gart.gart_layer_norm(x, y, g[:7]), lambda: gart.gart_layer_norm(x, y, g, g.half()),
           lambda: gart.gart_layer_norm(x.double(), y.double()), lambda: gart.gart_layer_norm(x[0], y[0]),
           lambda: gart.gart_layer_norm(x.t(), y.t()), lambda: gart.gart_layer_norm(x, y, x[:, 0]),
           lambda: gart.gart_layer_norm_backward(x, y.half()), lambda: gart.gart_layer_norm_backward(x, x, y, g[:5])]
    for f in bad:
        with pytest.raises(ValueError):
            f()
    worse = [lambda: gart.gart_layer_norm(x, y[:3]), lambda: gart.gart_layer_norm(x, y, eps=-1.0),
             lambda: gart.gart_layer_norm(x[1:], x[:3]), lambda: gart.gart_layer_norm(x, y[:1].expand(4, 8)),
             lambda: gart.gart_layer_norm_backward(x, y, x), lambda: gart.gart_layer_norm_backward(x, y[:3])]
    for f in worse:
        with pytest.raises(gart.GartError):
            f()
    torch.cuda.synchronize()
    assert (y == 5.0).all() and (x == 1.0).all()
