"""The appearance model with a layer norm ahead of its first layer, its matrices stepped by orthogonalised momentum:
every stage and every gradient against plain 64-bit forms, and a trainer's steps against the forms of both optimisers."""
import numpy as np
import pytest

import blocks_ref
import layer_norm_ref
import muon_ref
from paper_2608_17298_amd.scenes import make_scene, orbit_camera

pytestmark = pytest.mark.gpu
EPS = float(np.float32(1e-5))


def _f64(t):
    return t.cpu().double().numpy()


def _model(n, n_codes, sh_cols, seed=3, **kw):
    import torch
    from paper_2608_17298_amd.appearance import Appearance
    rng = np.random.default_rng(seed)
    codes = rng.integers(-1, n_codes, n)  # some have none
    a = Appearance(torch.from_numpy(codes).cuda(), n_codes, 2, sh_cols, seed=seed, norm=True, **kw)
    gen = torch.Generator("cuda").manual_seed(seed)
    a.params["w2"].normal_(0, 0.1, generator=gen)
    a.params["gain"].normal_(1, 0.2, generator=gen)
    a.params["shift"].normal_(0, 0.2, generator=gen)
    return a, codes, rng


@pytest.mark.parametrize("act,p,width", [("gelu", 0.1, 13), ("silu", 0.0, 32), ("none", 0.5, 8)])
def test_block_and_gradients(act, p, width):
    import torch
    a, codes, rng = _model(501, 20, 27, act=act, dropout=p, width=width, hidden=40, scale=0.7)
    base = torch.from_numpy(rng.standard_normal((501, 9, 3)).astype(np.float32)).cuda()
    a.forward(1, base, step=4)
    w = {k: _f64(v) for k, v in a.params.items()}
    e = _f64(a.e)
    want = layer_norm_ref.norm(e, w["gain"], w["shift"], EPS)
    assert (np.abs(_f64(a.n) - want) <= layer_norm_ref.norm_tolerance(e, w["gain"], w["shift"], EPS, "f32")).all()
    assert np.array_equal(_f64(a.n)[codes < 0], np.broadcast_to(w["shift"], (501, width))[codes < 0])
    h = blocks_ref.linear(_f64(a.n), w["w1"], w["b1"], None, act)
    tol = blocks_ref.linear_tolerance(_f64(a.n), w["w1"], w["b1"], None, act, "f32")
    assert (np.abs(_f64(a.h) - h) <= tol).all()
    # gradients of the whole block: sum g_sh sh by central differences in 64 bits
    g_sh = torch.from_numpy(rng.standard_normal((501, 9, 3)).astype(np.float32)).cuda()
    a.backward(g_sh, step=4)
    g64, scale, table = _f64(g_sh).reshape(501, 27), float(np.float32(0.7)), _f64(a.table[1])

    def loss(q, t):
        n = layer_norm_ref.norm(blocks_ref.embedding(t, codes, scale), q["gain"], q["shift"], EPS)
        d = blocks_ref.dropout(blocks_ref.linear(n, q["w1"], q["b1"], None, act), None, p, 3, 4)
        return (g64 * blocks_ref.linear(d, q["w2"], q["b2"], None, "none")).sum()

    for k in (*a.names, "table"):
        got = _f64(a.g_table if k == "table" else a.grads[k])
        v, vals = rng.standard_normal(got.shape), []
        for s in (1e-6, -1e-6):
            vals.append(loss(w, table + s * v) if k == "table" else loss({**w, k: w[k] + s * v}, table))
        # a chain of float32 stages of at most 501-term sums: 501 u of the terms' size; the codes' pass the norm's rstd
        raised = 1.0 / np.sqrt(e[codes >= 0].var(axis=1).min() + EPS) if k == "table" else 1.0
        size = np.abs(got * v).sum() + raised * np.abs(g64).sum()
        assert abs((got * v).sum() - (vals[0] - vals[1]) / 2e-6) <= 501 * blocks_ref.U32 * size, k


def _trainer(optimizer, norm, seed=1):
    import torch
    from paper_2608_17298_amd.appearance import Appearance
    from paper_2608_17298_amd.train import Trainer
    sc = make_scene("tiny", n=300, width=48, height=32)
    codes = torch.arange(sc.n, dtype=torch.int32, device="cuda") % 5
    model = Appearance(codes, 5, 2, 3 * (sc.sh_degree + 1) ** 2, width=8, hidden=16, seed=seed, norm=norm)
    gen = torch.Generator("cuda").manual_seed(2)
    targets = [torch.rand((32, 48, 3), device="cuda", generator=gen) for _ in range(2)]
    cams = [orbit_camera(48, 32, 0.0), orbit_camera(48, 32, 0.4)]
    return Trainer(sc, cams, targets, appearance=model, appearance_optimizer=optimizer, muon_decay=0.01), model


@pytest.mark.parametrize("norm", [True, False])
def test_trainer_steps_matrices_by_muon_and_the_rest_by_adam(norm):
    from paper_2608_17298_amd import train
    tr, model = _trainer("muon", norm)
    assert sorted(tr.muon) == ["w1", "w2"] and ("gain" in tr.am) == norm
    f = lambda v: float(np.float32(v))  # noqa: E731
    for step in range(1, 5):
        before = {k: (_f64(model.params[k]), _f64(tr.am[k]), _f64(tr.av[k]) if k in tr.av else None)
                  for k in model.names}
        assert np.isfinite(float(tr.step(step % 2)))
        for k in model.names:
            (p, m, v), g, got = before[k], _f64(model.grads[k]), _f64(model.params[k])
            if k in tr.muon:
                scale = max(1.0, p.shape[0] / p.shape[1]) ** 0.5
                args = (p, g, m, train.MUON_LR, train.MUON_MOMENTUM, 0.01, scale, True)
                want, m_want, o = muon_ref.muon(*args)
                plain = np.linalg.norm(muon_ref.muon(*args, dtype=np.float32)[2] - o)
                tol = 6 * blocks_ref.U32 * np.linalg.norm(want) + train.MUON_LR * scale * (
                    4 * plain + 16 * blocks_ref.U32 * np.linalg.norm(o))
                assert np.abs(_f64(tr.am[k]) - m_want).max() <= 2 * blocks_ref.U32 * np.abs(m_want).max()
            else:
                b1, b2 = f(0.9), f(0.999)
                m, v = b1 * m + (1 - b1) * g, b2 * v + (1 - b2) * g * g
                move = f(train.APPEARANCE_LR) * (m / (1 - b1 ** step)) / (np.sqrt(v / (1 - b2 ** step)) + f(1e-15))
                want = p - move
                # a few float32 roundings of each factor; 1 - b2^t keeps the rounding of b2's power over itself
                tol = np.sqrt(p.size) * (blocks_ref.U32 * np.abs(want).max() * 2
                                         + np.abs(move).max() * (20 + 4 / (1 - b2 ** step)) * blocks_ref.U32)
            assert np.linalg.norm(got - want) <= tol, (k, step)


def test_adam_is_as_before():
    """Without the norm, by Adam: the same parameters and no matrix stepped otherwise; unknown optimisers are refused."""
    tr, model = _trainer("adam", False)
    assert tr.muon == {} and model.names == ("w1", "b1", "w2", "b2") and model.n is model.e
    assert np.isfinite(float(tr.step(0)))
    with pytest.raises(ValueError):
        _trainer("sgd", False)


def test_norm_and_muon_in_a_graph():
    """A training step's part of the model (norm, gradients, orthogonalised step) captured and replayed as eager."""
    import torch
    from paper_2608_17298_amd import gart
    a, _, rng = _model(300, 12, 12, width=16, hidden=24)
    base = torch.zeros((300, 4, 3), device="cuda")
    g_sh = torch.from_numpy(rng.standard_normal((300, 4, 3)).astype(np.float32)).cuda()
    how = gart.gart_newton_schulz(3.4445, -4.775, 2.0315, 1e-7, 5)
    h = gart.gart_muon(0.02, 0.95, 0.0, 1.0, 1, how)
    start = {k: v.clone() for k, v in a.params.items()}
    m = {k: torch.zeros_like(a.params[k]) for k in ("w1", "w2")}
    scratch = torch.empty(max(gart.gart_muon_scratch_bytes(*a.params[k].shape) for k in m), dtype=torch.uint8,
                          device="cuda")

    def run():
        a.forward(0, base, step=1)
        a.backward(g_sh, step=1)
        for k in m:
            gart.gart_muon_step(a.params[k], a.grads[k], m[k], h, scratch)

    def reset():
        for k, v in start.items():
            a.params[k].copy_(v)
        for v in m.values():
            v.zero_()

    run()
    run()
    want = [a.params[k].clone() for k in a.names] + [v.clone() for v in m.values()]
    reset()
    run()  # eager work of the same tensors before and between
    reset()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        run()
    for _ in range(3):
        reset()
        graph.replay()
        graph.replay()
        torch.cuda.synchronize()
        for x, y in zip(want, [a.params[k] for k in a.names] + list(m.values())):
            assert torch.equal(x, y)
