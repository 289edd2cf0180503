"""The appearance model: its forward and gradients against plain 64-bit forms of the same block, and a training run on
views of one scene whose colours differ, which the scene's SH coefficients alone cannot fit."""
import numpy as np
import pytest

import blocks_ref as ref
from paper_2608_17298_amd.scenes import make_scene, orbit_camera

pytestmark = pytest.mark.gpu


def _model(n, n_codes, sh_cols, seed=3, **kw):
    import torch
    from paper_2608_17298_amd.appearance import Appearance
    rng = np.random.default_rng(seed)
    codes = rng.integers(-1, n_codes, n)  # some have none
    a = Appearance(torch.from_numpy(codes).cuda(), n_codes, 2, sh_cols, seed=seed, **kw)
    a.params["w2"].normal_(0, 0.1, generator=torch.Generator("cuda").manual_seed(seed))
    return a, codes, rng


@pytest.mark.parametrize("act,p", [("gelu", 0.1), ("silu", 0.0), ("none", 0.5)])
def test_block_and_gradients(act, p):
    """Every stage from the stored float32 input of that stage, so the bounds are the single operators'."""
    import torch
    a, codes, rng = _model(501, 20, 27, act=act, dropout=p, width=13, hidden=40, scale=0.7)
    f64 = lambda t: t.cpu().double().numpy()  # noqa: E731
    base = torch.from_numpy(rng.standard_normal((501, 9, 3)).astype(np.float32)).cuda()
    sh = a.forward(1, base, step=4)
    assert sh.shape == base.shape
    w = {k: f64(v) for k, v in a.params.items()}
    scale = float(np.float32(0.7))
    e = ref.embedding(f64(a.table[1]), codes, scale)
    assert (np.abs(f64(a.e) - e) <= 3 * ref.U32 * np.abs(e)).all()
    h = f64(a.h)
    assert (np.abs(h - ref.linear(f64(a.e), w["w1"], w["b1"], None, act))
            <= ref.linear_tolerance(f64(a.e), w["w1"], w["b1"], None, act, "f32")).all()
    d = ref.dropout(h, None, p, 3, 4)
    assert (np.abs(f64(a.d) - d) <= ref.dropout_tolerance(h, None, p, "f32", d)).all()
    b64 = f64(base).reshape(501, 27)
    assert (np.abs(f64(a.sh) - ref.linear(f64(a.d), w["w2"], w["b2"], b64, "none"))
            <= ref.linear_tolerance(f64(a.d), w["w2"], w["b2"], b64, "none", "f32")).all()
    # gradients of the whole block: sum g_sh sh by central differences in 64 bits
    g_sh = torch.from_numpy(rng.standard_normal((501, 9, 3)).astype(np.float32)).cuda()
    a.backward(g_sh, step=4)
    g64 = f64(g_sh).reshape(501, 27)

    def loss(p64, table):
        h = ref.linear(ref.embedding(table, codes, scale), p64["w1"], p64["b1"], None, act)
        d = ref.dropout(h, None, p, 3, 4)
        return (g64 * ref.linear(d, p64["w2"], p64["b2"], None, "none")).sum()

    table = f64(a.table[1])
    for k in ("w1", "b1", "w2", "b2", "table"):
        got = f64(a.g_table if k == "table" else a.grads[k])
        v = rng.standard_normal(got.shape)
        vals = []
        for s in (1e-6, -1e-6):
            q, t = dict(w), table
            if k == "table":
                t = table + s * v
            else:
                q[k] = w[k] + s * v
            vals.append(loss(q, t))
        # a chain of float32 stages of at most 501-term sums: 501 u of the terms' size, far above the differences' error
        size = np.abs(got * v).sum() + np.abs(g64).sum()
        assert abs((got * v).sum() - (vals[0] - vals[1]) / 2e-6) <= 501 * ref.U32 * size, k


def test_evaluation_drops_nothing():
    import torch
    a, _, rng = _model(200, 7, 12, dropout=0.5)
    base = torch.zeros((200, 4, 3), device="cuda")
    a.forward(0, base, train=False)
    assert torch.equal(a.d, a.h)


def test_training_fits_views_of_different_colour():
    import torch
    from paper_2608_17298_amd import gart
    from paper_2608_17298_amd.appearance import Appearance
    from paper_2608_17298_amd.train import Trainer
    sc = make_scene("tiny", n=800, width=64, height=48)
    cams = [orbit_camera(64, 48, 0.0), orbit_camera(64, 48, 0.0)]
    g = gart.Gaussians.from_scene(sc)
    st = gart.make_settings(sc.tile)
    frame = gart.prepare(g, gart.make_camera(cams[0]), st)
    image = torch.empty((48, 64, 3), device="cuda")
    gart.gart_forward(g, gart.make_camera(cams[0]), st, frame, image)
    tint = [torch.tensor(t, device="cuda") for t in ([1.0, 0.6, 0.4], [0.4, 0.7, 1.0])]
    targets = [(image * t).contiguous() for t in tint]  # one camera, two colours: no scene fits both
    codes = torch.zeros(sc.n, dtype=torch.int32, device="cuda")
    last = {}
    for name in ("scene", "appearance"):
        model = Appearance(codes, 1, 2, g.sh[0].numel(), width=8, hidden=16, dropout=0.1, seed=1) \
            if name == "appearance" else None
        tr = Trainer(sc, cams, targets, appearance=model, appearance_lr=1e-2)
        losses = [float(tr.step(i % 2)) for i in range(120)]
        assert np.isfinite(losses).all()
        last[name] = np.mean(losses[-10:])
        first = np.mean(losses[:2])
    # the scene alone can only meet both colours half way (their distance is spread over every step);
    # the model has a row for each view
    assert last["appearance"] < 0.6 * last["scene"] and last["appearance"] < 0.5 * first


def test_trainer_refuses_a_model_of_another_scene():
    import torch
    from paper_2608_17298_amd.appearance import Appearance
    from paper_2608_17298_amd.train import Trainer
    sc = make_scene("tiny", n=50, width=32, height=32)
    model = Appearance(torch.zeros(49, dtype=torch.int32, device="cuda"), 1, 1, 3)
    with pytest.raises(ValueError):
        Trainer(sc, [orbit_camera(32, 32, 0.0)], [torch.zeros((32, 32, 3), device="cuda")], appearance=model)
