"""Orthogonalised matrices and momentum steps on the GPU against plain 64-bit forms: every type, flat, tall and square
ones from one element up, odd and strided, rank-deficient, zero and non-finite, other coefficients, streams, graphs."""
import numpy as np
import pytest

import blocks_ref
import muon_ref as ref
from test_gpu_blocks import GUARD, TYPES, _Out, _inside, _mat, _scratch, _torch, _within

pytestmark = pytest.mark.gpu

# sizes on both sides of the borders between the kernels, and of those of small tiles; the large tiles': muon_sizes.py
SIZES = [(1, 1), (1, 7), (5, 1), (2, 3), (3, 2), (16, 16), (17, 33), (33, 17), (48, 64), (64, 32), (32, 64), (65, 63),
         (64, 65), (7, 300), (300, 7), (1, 4096), (4096, 1), (100, 129), (129, 100), (128, 128), (96, 200), (200, 96),
         (40, 1000), (1000, 40), (255, 255), (256, 130), (130, 700), (700, 130), (512, 300), (300, 512), (500, 1500),
         (1500, 500), (640, 640), (64, 3000), (2600, 65)]


def _how(gart, steps=5, abc=ref.COEFFICIENTS, eps=ref.EPS):
    return gart.gart_newton_schulz(*abc, eps, steps)


def _gradient(rng, rows, cols, kind="decay"):
    """A few strong directions and ever weaker ones; "deficient": a third of the rank; "normal": all alike."""
    k = min(rows, cols)
    if kind == "normal":
        return rng.standard_normal((rows, cols)) * 1e-3
    r = max(1, k // 3) if kind == "deficient" else k
    return (rng.standard_normal((rows, r)) * np.logspace(0, -2, r)) @ rng.standard_normal((r, cols)) * 1e-3


def _device(values, dtype, pad=0):
    import torch
    rows, cols = values.shape
    t = torch.full((rows, cols + pad), GUARD, dtype=_torch(dtype), device="cuda")[:, :cols]
    t.copy_(torch.from_numpy(values))
    return t, t.cpu().double().numpy()


def _orthogonalize(x, dtype, pad=0, **kw):
    from paper_2608_17298_amd import gart
    y = _Out(*x.shape, dtype, pad)
    gart.gart_orthogonalize(x, y.t, _how(gart, **kw),
                            _scratch(gart.gart_orthogonalize_scratch_bytes(*x.shape, x.dtype)))
    return y.value()


def _exact_as_float32(got, x64, dtype, **kw):
    """In the 2-norm at most four times as far off as the same steps in float32 elementary operations (and a float32
    rounding), besides the result's own rounding."""
    want = ref.orthogonalize(x64, **kw)
    plain = np.linalg.norm(ref.orthogonalize(x64, dtype=np.float32, **kw) - want)
    size = np.linalg.norm(want)
    off = np.linalg.norm(got - want)
    assert off <= 4.0 * plain + (8.0 * blocks_ref.U32 + (0.0 if dtype == "f32" else 1.01 * blocks_ref.U[dtype])) * size, \
        (off / size, plain / size)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("rows,cols", SIZES)
@pytest.mark.parametrize("kind,pad", [("decay", 0), ("deficient", 3), ("normal", 8)])
def test_orthogonalize(rows, cols, dtype, kind, pad):
    rng = np.random.default_rng(rows + 3 * cols)
    x, x64 = _device(_gradient(rng, rows, cols, kind), dtype, pad)
    got = [_orthogonalize(x, dtype, 2 * pad) for _ in range(2)]
    assert np.array_equal(got[0], got[1])  # deterministic
    _exact_as_float32(got[0], x64, dtype)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("rows,cols", SIZES)
def test_one_step_element_by_element(rows, cols, dtype):
    """One step's bound is tight enough to find a wrong or missing product of low parts."""
    rng = np.random.default_rng(rows * 5 + cols)
    x, x64 = _device(_gradient(rng, rows, cols, "normal"), dtype, 1)
    got = _orthogonalize(x, dtype, 3, steps=1)
    _within(got, ref.orthogonalize(x64, 1), ref.one_step_tolerance(x64, dtype))


@pytest.mark.parametrize("steps", [1, 2, 3, 4, 6, 7, 8, 12])
@pytest.mark.parametrize("rows,cols", [(30, 50), (50, 30), (90, 400), (400, 90), (300, 320), (200, 900), (900, 200)])
def test_steps(rows, cols, steps):
    rng = np.random.default_rng(steps)
    x, x64 = _device(_gradient(rng, rows, cols), "f32")
    _exact_as_float32(_orthogonalize(x, "f32", steps=steps), x64, "f32", steps=steps)


@pytest.mark.parametrize("rows,cols", [(30, 50), (100, 128), (300, 200), (1100, 1000)])
def test_most_steps(rows, cols):
    """64 steps of polynomials that settle at 1: the result's singular values are 1, as nearly as float32's steps'."""
    rng = np.random.default_rng(rows)
    x, x64 = _device(rng.standard_normal((rows, cols)), "f32")
    abc = (1.875, -1.25, 0.375)
    got = _orthogonalize(x, "f32", steps=64, abc=abc)
    _exact_as_float32(got, x64, "f32", steps=64, abc=list(abc))


def test_more_tiles_of_rows_than_a_grid_is_high():
    """Four million rows of two columns: 65626 tiles of 64."""
    import torch
    from paper_2608_17298_amd import gart
    if torch.cuda.mem_get_info()[0] < 12 << 30:
        pytest.skip("needs 9 GB of device memory")
    rng = np.random.default_rng(8)
    x, x64 = _device(rng.standard_normal((4_200_001, 2)).astype(np.float32), "bf16")
    y = torch.empty_like(x)
    gart.gart_orthogonalize(x, y, _how(gart), _scratch(gart.gart_orthogonalize_scratch_bytes(*x.shape, x.dtype)))
    want = ref.orthogonalize(x64)
    got = y.cpu().double().numpy()
    # sums of 4.2 million terms, in parts of at most 131250 blocks of 32: their relative error stays below 2^-8 / 4
    assert (np.abs(got - want) <= 1.25 * blocks_ref.U["bf16"] * np.abs(want) + 1e-9).all()


@pytest.mark.parametrize("abc", [(1.5, -0.5, 0.0), (1.875, -1.25, 0.375), (2.0, -1.5, 0.5), (0.5, 0.0, 0.0),
                                 (0.8, 0.0, 0.2), (-3.0, 4.0, -1.5), (0.0, 0.0, 0.0), (4.0, 0.0, 0.0)])
@pytest.mark.parametrize("rows,cols", [(20, 30), (70, 300), (300, 200), (400, 1000)])
def test_coefficients(rows, cols, abc):
    rng = np.random.default_rng(rows)
    x, x64 = _device(_gradient(rng, rows, cols), "f32")
    got = _orthogonalize(x, "f32", abc=abc, steps=4)
    _exact_as_float32(got, x64, "f32", abc=[float(np.float32(v)) for v in abc], steps=4)


@pytest.mark.parametrize("rows,cols", [(20, 40), (96, 33), (150, 600), (520, 260)])
def test_singular_vectors_stay(rows, cols):
    """Against the definition itself: the singular values of x over its norm, each taken through the polynomial."""
    rng = np.random.default_rng(cols)
    x, x64 = _device(rng.standard_normal((rows, cols)), "f32")
    u, s, v = np.linalg.svd(x64, full_matrices=False)
    s = s / (np.sqrt((s ** 2).sum()) + ref.EPS)
    want = (u * ref.singular_values(s)) @ v
    got = _orthogonalize(x, "f32")
    plain = np.linalg.norm(ref.orthogonalize(x64, dtype=np.float32) - want)
    assert np.linalg.norm(got - want) <= 4.0 * plain + 8.0 * blocks_ref.U32 * np.linalg.norm(want)


@pytest.mark.parametrize("scale", [1e-30, 1e-12, 1e6, 1e18, 1e30])
@pytest.mark.parametrize("rows,cols", [(40, 70), (70, 300), (300, 150)])
def test_sizes_of_the_elements(rows, cols, scale):
    """Only eps knows how large x is: squares neither overflow nor vanish."""
    rng = np.random.default_rng(rows)
    x, x64 = _device(rng.standard_normal((rows, cols)) * scale, "f32")
    _exact_as_float32(_orthogonalize(x, "f32"), x64, "f32")


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("rows,cols", [(1, 1), (40, 30), (70, 300), (300, 200), (500, 600)])
def test_zero_matrix(rows, cols, dtype):
    import torch
    x = torch.zeros((rows, cols), dtype=_torch(dtype), device="cuda")
    assert (_orthogonalize(x, dtype) == 0).all()
    assert np.isnan(_orthogonalize(x, dtype, eps=0.0)).all()


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("value", [float("nan"), float("inf"), -float("inf")])
@pytest.mark.parametrize("rows,cols", [(1, 1), (3, 5), (48, 64), (70, 300), (300, 70), (300, 200), (500, 600)])
def test_nonfinite(rows, cols, value, dtype):
    rng = np.random.default_rng(rows)
    x, _ = _device(_gradient(rng, rows, cols), dtype)
    x[rows // 2, cols - 1] = value
    assert np.isnan(_orthogonalize(x, dtype)).all()


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("rows,cols,pad", [(1, 1, 3), (48, 64, 1), (64, 33, 8), (70, 300, 3), (300, 70, 1), (301, 200, 8),
                                           (500, 700, 0)])
def test_uses_nothing_around_its_inputs(rows, cols, pad, dtype):
    """NaN around x: the result is that with zeros there, bit for bit; likewise y over x, and scratch full of NaN."""
    import torch
    from paper_2608_17298_amd import gart
    rng = np.random.default_rng(rows)
    v = _gradient(rng, rows, cols)
    got = [_orthogonalize(_inside(v, dtype, pad, around), dtype, pad) for around in (0.0, float("nan"))]
    assert np.isfinite(got[0]).all() and np.array_equal(got[0], got[1])
    x = _inside(v, dtype, pad, float("nan"))
    s = torch.zeros(gart.gart_orthogonalize_scratch_bytes(rows, cols, x.dtype), dtype=torch.uint8, device="cuda")
    gart.gart_orthogonalize(x, x, _how(gart), s)
    assert np.array_equal(x.cpu().double().numpy(), got[0])


def test_repeated_row():
    """One row repeated (stride 0) has one singular value, sqrt(rows) |row| over its norm: 1."""
    rng = np.random.default_rng(0)
    row, r64 = _mat(rng, 1, 50, "f32")
    got = _orthogonalize(row.expand(20, 50), "f32")
    want = np.repeat(r64 / np.linalg.norm(r64), 20, 0) / np.sqrt(20) * ref.singular_values(1.0)
    # five steps of relative errors 40 u or less each, none of which the slope at s near 1 raises (|p'| < 4)
    assert np.abs(got - want).max() <= 5 * 40 * 4 * blocks_ref.U32 * np.abs(want).max()


# ---- the momentum step ---------------------------------------------------------------
H = dict(lr=0.02, momentum=0.95, decay=0.01)


def _muon_h(gart, scale, nesterov, steps=5, **kw):
    h = {**H, **kw}
    return gart.gart_muon(h["lr"], h["momentum"], h["decay"], scale, int(nesterov), _how(gart, steps))


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("rows,cols", SIZES)
@pytest.mark.parametrize("nesterov,pad,scale", [(True, 0, 1.0), (False, 3, 1.7)])
def test_muon_step(rows, cols, dtype, nesterov, pad, scale):
    import torch
    from paper_2608_17298_amd import gart
    rng = np.random.default_rng(rows + 7 * cols)
    f = lambda v: float(np.float32(v))  # noqa: E731
    p0, p64 = _device(rng.standard_normal((rows, cols)) * cols ** -0.5, dtype, pad)
    g, g64 = _device(_gradient(rng, rows, cols), dtype, pad)
    m0, m64 = _device(_gradient(rng, rows, cols) * 4, "f32", 2 * pad)
    scratch = _scratch(gart.gart_muon_scratch_bytes(rows, cols, p0.dtype))
    runs = []
    for _ in range(2):
        p, m = _Out(rows, cols, dtype, pad), _Out(rows, cols, "f32", pad)
        p.t.copy_(p0)
        m.t.copy_(m0)
        gart.gart_muon_step(p.t, g, m.t, _muon_h(gart, scale, nesterov), scratch)
        runs.append((p.value(), m.value()))
    assert np.array_equal(runs[0][0], runs[1][0]) and np.array_equal(runs[0][1], runs[1][1])
    args = (p64, g64, m64, H["lr"], H["momentum"], H["decay"], scale, nesterov)
    want, m_want, o = ref.muon(*args)
    _, _, o32 = ref.muon(*args, dtype=np.float32)
    _within(runs[0][1], m_want, 1.01 * blocks_ref.U32 * np.abs(m_want) + blocks_ref.TINY["f32"])
    step, plain = f(H["lr"]) * f(scale), np.linalg.norm(o32 - o)
    tol = 1.01 * blocks_ref.U[dtype] * np.linalg.norm(want) + 4 * blocks_ref.U32 * (
        np.linalg.norm(p64) + step * np.linalg.norm(o)) + step * (4 * plain + 8 * blocks_ref.U32 * np.linalg.norm(o))
    assert np.linalg.norm(runs[0][0] - want) <= tol
    # and no element is off by more than all of that
    assert (np.abs(runs[0][0] - want) <= 1.01 * blocks_ref.U[dtype] * np.abs(want) + blocks_ref.TINY[dtype]
            + 4 * blocks_ref.U32 * np.abs(p64) + step * (4 * plain + 16 * blocks_ref.U32 * np.linalg.norm(o))).all()
    assert torch.equal(g, g.clone())


def test_muon_steps_in_a_row():
    """Ten steps with their own gradients: the momentum is carried, and the parameters stay with the 64-bit ones."""
    from paper_2608_17298_amd import gart
    rng = np.random.default_rng(1)
    rows, cols = 60, 44
    p, p64 = _device(rng.standard_normal((rows, cols)) * 0.1, "f32")
    m, m64 = _device(np.zeros((rows, cols)), "f32")
    s = _scratch(gart.gart_muon_scratch_bytes(rows, cols))
    for _ in range(10):
        g, g64 = _device(_gradient(rng, rows, cols, "normal"), "f32")
        gart.gart_muon_step(p, g, m, _muon_h(gart, 1.0, True), s)
        p64, m64, o = ref.muon(p64, g64, m64, H["lr"], H["momentum"], H["decay"], 1.0, True)
    # rounding of m (u a step) is raised at most |p5'(0)| = 3.4445^5 = 485 fold in o; ten steps add up
    tol = 10 * (0.02 * 485 * 10 * blocks_ref.U32 * np.linalg.norm(o) + 4 * blocks_ref.U32 * np.linalg.norm(p64))
    assert np.linalg.norm(p.cpu().double().numpy() - p64) <= tol


def test_muon_first_step_without_momentum_or_decay():
    """From m = 0 with momentum 0: m is the gradient, and param moves by lr scale orthogonalize(gradient)."""
    import torch
    from paper_2608_17298_amd import gart
    rng = np.random.default_rng(2)
    g, _ = _device(_gradient(rng, 40, 60), "f32")
    p, m = torch.zeros_like(g), torch.zeros_like(g)
    gart.gart_muon_step(p, g, m, _muon_h(gart, 1.0, True, momentum=0.0, decay=0.0, lr=0.5),
                        _scratch(gart.gart_muon_scratch_bytes(40, 60)))
    assert torch.equal(m, g)
    o = _orthogonalize(g, "f32")
    assert np.array_equal(p.cpu().double().numpy(), -0.5 * o)


def test_offsets_beyond_32_bits():
    """Rows 2^22 elements apart, 1040 of them: element offsets pass 2^32."""
    import torch
    from paper_2608_17298_amd import gart
    rows, step, cols = 1040, 1 << 22, 70
    if torch.cuda.mem_get_info()[0] < 60 << 30:
        pytest.skip("needs 52 GB of device memory")
    rng = np.random.default_rng(3)
    s = _scratch(gart.gart_muon_scratch_bytes(rows, cols, torch.bfloat16))
    near = [_device(_gradient(rng, rows, cols), d)[0] for d in ("bf16", "bf16", "f32")]
    far = []
    for t in near:
        b = torch.empty((rows - 1) * step + cols, dtype=t.dtype, device="cuda")
        far.append(b.as_strided((rows, cols), (step, 1)))
        far[-1].copy_(t)
    for p, g, m in (near, far):
        gart.gart_muon_step(p, g, m, _muon_h(gart, 1.0, True), s)
        gart.gart_orthogonalize(p, g, _how(gart), s)
    for a, b in zip(near, far):
        assert torch.equal(a, b)


def _calls(rows, cols, dtype="bf16"):
    import torch
    from paper_2608_17298_amd import gart
    rng = np.random.default_rng(4)
    g, p0, m0 = (_device(_gradient(rng, rows, cols), d)[0] for d in (dtype, dtype, "f32"))
    p, m, y = torch.empty_like(p0), torch.empty_like(m0), torch.empty_like(p0)
    s = _scratch(gart.gart_muon_scratch_bytes(rows, cols, g.dtype))

    def run(stream=None):
        gart.gart_muon_step(p, g, m, _muon_h(gart, 1.0, True), s, stream=stream)
        gart.gart_orthogonalize(p, y, _how(gart), s, stream=stream)

    def reset():
        p.copy_(p0)
        m.copy_(m0)
        y.fill_(GUARD)
        torch.cuda.synchronize()

    return run, reset, [p, m, y]


@pytest.mark.parametrize("rows,cols", [(48, 64), (40, 1000), (300, 200), (300, 1300)])
def test_another_stream_and_graphs(rows, cols):
    """On a side stream, and captured once and replayed four times with other work between."""
    import torch
    run, reset, outs = _calls(rows, cols)
    reset()
    run()
    torch.cuda.synchronize()
    want = [t.clone() for t in outs]
    reset()
    side = torch.cuda.Stream()
    run(side)
    side.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(outs, want))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        run()
    for _ in range(4):
        reset()
        (torch.randn((512, 512), device="cuda") * 2.0).sum().item()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(outs, want))


def test_refusals_on_tensors():
    """Tensors of the wrong kind are refused before the library is called, and nothing is written."""
    import torch
    from paper_2608_17298_amd import gart
    x, g = torch.ones((4, 8), device="cuda"), torch.ones((4, 8), device="cuda")
    y = torch.full((4, 8), 5.0, device="cuda")
    s = _scratch(gart.gart_muon_scratch_bytes(4, 8))
    how, h = _how(gart), _muon_h(gart, 1.0, True)
    bad = [lambda: gart.gart_orthogonalize(x.cpu(), y, how, s), lambda: gart.gart_orthogonalize(x, y.half(), how, s),
           lambda: gart.gart_orthogonalize(x[0], y[0], how, s), lambda: gart.gart_orthogonalize(x.t(), y.t(), how, s),
           lambda: gart.gart_orthogonalize(x.double(), y.double(), how, s),
           lambda: gart.gart_orthogonalize(x, y, how, s.cpu()),
           lambda: gart.gart_muon_step(x, g, y.bfloat16(), h, s), lambda: gart.gart_muon_step(x, g.half(), y, h, s),
           lambda: gart.gart_muon_step(x, g, y.cpu(), h, s)]
    for f in bad:
        with pytest.raises(ValueError):
            f()
    worse = [lambda: gart.gart_orthogonalize(x, y[:3], how, s), lambda: gart.gart_orthogonalize(x, y, how, None),
             lambda: gart.gart_orthogonalize(x, y, how, s[:-16]), lambda: gart.gart_muon_step(x, x, y, h, s),
             lambda: gart.gart_muon_step(x, g[:, :7], y, h, s), lambda: gart.gart_muon_step(x[:1].expand(4, 8), g, y, h, s)]
    for f in worse:
        with pytest.raises(gart.GartError):
            f()
    torch.cuda.synchronize()
    assert (y == 5.0).all() and (x == 1.0).all() and (g == 1.0).all()
