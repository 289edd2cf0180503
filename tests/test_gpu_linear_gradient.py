"""The linear layer's gradient in 16 bits: dz = dl act'(z) enters its products in more than the type's bits, so the
results are float32's rounded once, also beyond float16's range and among its smallest numbers, and infinities stay
infinities.  Every kernel that takes part: streams, tiles, parts of sums, few rows."""
import numpy as np
import pytest

import blocks_ref as ref
from test_gpu_blocks import _Out, _mat, _scratch, _torch, _vec, _within

pytestmark = pytest.mark.gpu

# dz is the sum of two numbers of the type, the first one cut off (bf16: 7 bits behind the point, f16: 10), the second
# rounded (bf16: 2^-8 of what is left) or cut off (f16: 2^-10), with float16's smallest numbers 2^-33 apart
PARTS = dict(bf16=2.0 ** -15, f16=2.0 ** -20)
LEAST = dict(bf16=2.0 ** -126, f16=2.0 ** -33)

STREAMS = [(300, 24, 20), (1000, 64, 48), (2051, 64, 128), (700, 200, 100), (129, 128, 256), (513, 30, 250),
           (400, 9, 17)]
TILES = [(700, 520, 130), (300, 300, 40), (2000, 300, 500), (90, 1000, 1000), (40, 1500, 700), (3592, 64, 4040),
         (20000, 272, 40), (100, 4040, 72), (257, 513, 259)]

FEW_ROWS = [(10, 1500, 700), (20, 1500, 700), (50, 900, 700)]


def _tolerance(x, w, b, dl, act, dtype):
    """float32's own errors (blocks_ref.linear_grads_tolerance), those of dz's parts, twice as many terms, one
    rounding of the result."""
    z = x @ w.T + (0.0 if b is None else b)
    dz = np.abs(dl * ref.act_grad(z, act))
    e = PARTS[dtype] * dz + LEAST[dtype]
    own = ref.linear_grads_tolerance(x, w, b, dl, act, "f32")
    gx, gw, gb = ref.linear_grads(x, w, b, dl, act)
    m, n = dz.shape
    more = (e @ np.abs(w) + 1.2 * ref.U32 * n * (dz + e) @ np.abs(w),
            e.T @ np.abs(x) + 1.2 * ref.U32 * m * (dz + e).T @ np.abs(x), 0.0)
    return [o + p + 1.01 * ref.U[dtype] * np.abs(g) + ref.TINY[dtype] for o, p, g in zip(own, more, (gx, gw, gb))]


def _gradients(x, w, dl, b, act, dtype, pad=0):
    from paper_2608_17298_amd import gart
    (m, k), n = x.shape, w.shape[0]
    out = _Out(m, k, dtype, pad), _Out(n, k, dtype, pad), _Out(1, n, dtype, 0)
    gart.gart_linear_backward(x, w, dl, out[0].t, out[1].t, out[2].t.reshape(-1), b, act,
                              _scratch(gart.gart_linear_backward_scratch_bytes(m, k, n, _torch(dtype), act)))
    return out[0].value(), out[1].value(), out[2].value()[0]


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("m,k,n", STREAMS + TILES + FEW_ROWS)
@pytest.mark.parametrize("act,pad", [("silu", 0), ("gelu", 3)])
def test_gradient_rounds_once(m, k, n, act, pad, dtype):
    rng = np.random.default_rng(m + 3 * k + 5 * n)
    (x, x64), (w, w64) = _mat(rng, m, k, dtype, pad), _mat(rng, n, k, dtype, pad, k ** -0.5)
    (b, b64), (dl, d64) = _vec(rng, n, dtype), _mat(rng, m, n, dtype, pad)
    got = _gradients(x, w, dl, b, act, dtype, pad)
    for g, want, tol in zip(got, ref.linear_grads(x64, w64, b64, d64, act), _tolerance(x64, w64, b64, d64, act, dtype)):
        _within(g, want, tol)


@pytest.mark.parametrize("m,k,n", [(16, 24, 20), (300, 24, 20), (700, 200, 100), (700, 520, 130), (40, 1500, 700),
                                   (90, 1000, 1000)])
@pytest.mark.parametrize("size", ["large", "small, large x", "small, large w"])
def test_float16_gradient_beyond_the_type(m, k, n, size):
    """dl at float16's upper end, where slopes above 1 take dz past it, and among its subnormals, where it is a few
    units; the results are in the type's range."""
    rng = np.random.default_rng(m + n)
    (x, x64), (w, w64) = _mat(rng, m, k, "f16"), _mat(rng, n, k, "f16", 0, k ** -0.5)
    b, b64 = _vec(rng, n, "f16")
    if size == "large":
        x, w = (x * 2.0 ** -9).contiguous(), (w * 2.0 ** -9).contiguous()
        b = b * 0.1 + 1.5  # gelu's slope is largest, 1.13, about there
        dl, _ = _mat(rng, m, n, "f16", 0, 500.0)
        dl[:, ::3] = 65000.0
        dl[:, 1::3] = -64000.0
    else:
        dl, _ = _mat(rng, m, n, "f16", 0, 2.0 ** -21)
        up = 256.0 if size == "small, large x" else 1.0 / 256.0  # z is the same
        x, w = (x * up).contiguous(), (w / up).contiguous()
    x64, w64, b64, d64 = (t.cpu().double().numpy() for t in (x, w, b, dl))
    got = _gradients(x, w, dl, b, "gelu", "f16")
    want = ref.linear_grads(x64, w64, b64, d64, "gelu")
    for g, a, tol in list(zip(got, want, _tolerance(x64, w64, b64, d64, "gelu", "f16")))[:2]:
        a = np.where(np.abs(a) >= 65520.0, np.copysign(np.inf, a), a)  # what the type holds
        sure = np.isfinite(a) & (np.abs(a) + tol < 65504.0)
        assert sure.mean() > 0.5
        assert np.isfinite(g[sure]).all()
        _within(g[sure], a[sure], tol[sure])


@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("act", ["silu", "gelu"])
@pytest.mark.parametrize("m,k,n", [(3, 9, 5), (40, 1500, 700), (300, 24, 20), (700, 70, 33), (300, 300, 40),
                                   (2000, 32, 64), (700, 520, 130)])
def test_infinite_gradients_and_inputs_stay_infinite(m, k, n, act, dtype):
    """An infinite dl[r, j] gives infinities of W's signs in g_x[r] and of x's in g_weight[j]; an infinite x[r, c]
    gives g_weight[j, c] infinities of dl's signs for the outputs whose slope is 1 (0 times infinity for the others)."""
    import torch
    rng = np.random.default_rng(m + k + n)
    t, r, j, c = _torch(dtype), m // 2, n - 1, k // 3
    sign = lambda *s: torch.from_numpy(np.where(rng.random(s) < 0.5, -1.0, 1.0)).to(t).cuda()  # noqa: E731
    x, w, dl = sign(m, k), sign(n, k), sign(m, n)
    w *= 2.0 ** -6
    dl[r, j] = float("inf")
    gx, gw, gb = _gradients(x, w, dl, None, act, dtype)
    # the slope at (r, j) is positive: |z| <= k / 64, unless many inputs agree
    z = float((x[r].double() * w[j].double()).sum())
    if act == "silu" and z > -1.0 or act == "gelu" and z > -0.7:
        assert np.array_equal(gx[r], np.where(w[j].cpu().double().numpy() > 0, np.inf, -np.inf))
        assert np.array_equal(gw[j], np.where(x[r].cpu().double().numpy() > 0, np.inf, -np.inf))
        assert gb[j] == np.inf
    assert np.isfinite(np.delete(gx, r, 0)).all() and np.isfinite(np.delete(gw, j, 0)).all()
    dl[r, j] = 1.0
    x[r, c] = float("inf")
    gw = _gradients(x, w, dl, None, act, dtype)[1]
    up = w[:, c].cpu().double().numpy() > 0
    want = np.where(dl[r].cpu().double().numpy() > 0, np.inf, -np.inf)
    assert np.array_equal(gw[up, c], want[up]) and np.isnan(gw[~up, c]).all()
    assert np.isfinite(np.delete(gw, c, 1)).all()


@pytest.mark.parametrize("act", ["silu", "gelu"])
@pytest.mark.parametrize("rows", [1, 70])
def test_slopes_are_exact_to_a_few_roundings(act, rows):
    """act'(z) of single pre-activations, which are exact: g + z u' g (1 - g) with g = 1 / (1 + exp(-u)).  A few
    roundings of each term; the exponent's own, which moves exp(-u) by about |u| u32, moves g and 1 - g by g (1 - g)
    of it."""
    import torch
    from paper_2608_17298_amd import gart
    z = np.concatenate([np.linspace(-12.0, 12.0, 2001), np.linspace(-100.0, 100.0, 401)]).astype(np.float32)
    x, w = torch.zeros((rows, 3), device="cuda"), torch.zeros((len(z), 3), device="cuda")
    x[:, 0], w[:, 0] = 1.0, torch.from_numpy(z).cuda()
    dl = torch.zeros((rows, len(z)), device="cuda")
    dl[0] = 1.0
    gb = torch.empty(len(z), device="cuda")
    gart.gart_linear_backward(x, w, dl, None, None, gb, None, act,
                              _scratch(gart.gart_linear_backward_scratch_bytes(rows, 3, len(z), torch.float32, act)))
    z = z.astype(np.float64)
    c = 2.0 * np.sqrt(2.0 / np.pi)
    u = z if act == "silu" else c * (z + 0.044715 * z ** 3)
    du = np.ones_like(z) if act == "silu" else c * (1.0 + 3.0 * 0.044715 * z ** 2)
    e = np.exp(-np.abs(u))
    g, h = np.where(u > 0, 1.0, e) / (1.0 + e), np.where(u > 0, e, 1.0) / (1.0 + e)  # gate, and 1 - gate
    want = g + z * du * g * h
    tol = ref.U32 * (6.0 * g + 12.0 * np.abs(z * du) * g * h + (4.0 * np.abs(u) + 8.0) * g * h * (1.0 + np.abs(z * du)))
    _within(gb.cpu().double().numpy(), want, tol + 1e-35)
