"""Operator cases: the learned blocks in front of the Gaussians' parameters, each operator on its own.

An appearance model looks a code up for every Gaussian (a row of a table, shared by a cluster of them and chosen by the
view), turns it into SH coefficients with a small feed-forward block with dropout, and takes the gradient of the SH
coefficients back into the block's weights and the table.  A case names one call of it:

  embedding           gart_embedding: out[i] = scale * table[ids[i]], zero where the id is outside the table
  embedding_backward  gart_embedding_backward: the table's gradient, summed over the ids
  linear              gart_linear: y = act(x W^T + bias) + residual
  linear_backward     gart_linear_backward: gradients of x, W and bias from dL/dy (the pre-activation is not stored)
  dropout             gart_dropout: residual + x * keep / (1 - p), keep from a counter-based generator; without a
                      residual it is also the operator's gradient
"""
from __future__ import annotations

import math

import numpy as np
import torch

own = False

_TYPES = dict(f32=torch.float32, bf16=torch.bfloat16, f16=torch.float16)


def _embedding(name, do, n, dim, vocab, dtype, ids="int64", skew=True, absent=False, pad=0):
    return dict(name=name, do=do, n=n, dim=dim, vocab=vocab, dtype=dtype, ids=ids, skew=skew, absent=absent, pad=pad)


def _linear(name, do, rows, inputs, outputs, dtype, act, bias=True, residual=False, pad=0):
    return dict(name=name, do=do, rows=rows, inputs=inputs, outputs=outputs, dtype=dtype, act=act, bias=bias,
                residual=residual, pad=pad)


def _dropout(name, rows, cols, dtype, p, residual, pad=0):
    return dict(name=name, do="dropout", rows=rows, cols=cols, dtype=dtype, p=p, residual=residual, pad=pad)


def listed():
    return [
        # one code is shown: the latency of a call
        _embedding("lookup-one", "embedding", 1, 32, 4096, "f32", skew=False),
        # SH rows of degree 3 from a table of shared colours, one for each Gaussian of the 1m workload
        _embedding("lookup-1m-sh", "embedding", 1_000_000, 48, 65_536, "f32", ids="int32", absent=True),
        # gradient of a table of cluster codes: few rows, some of them used by many thousands of Gaussians
        _embedding("codes-grad-1m", "embedding_backward", 1_000_000, 64, 4096, "bf16"),
        # gradient of a large vocabulary from a batch of tokens: odd sizes, most rows unused
        _embedding("vocab-grad", "embedding_backward", 8191, 1023, 50_021, "f16", absent=True),
        # one row through a wide layer: a single token is served
        _linear("layer-one-row", "linear", 1, 1024, 4096, "bf16", "silu"),
        # first layer of the block over the Gaussians of the 1m workload
        _linear("layer-1m-hidden", "linear", 1_000_000, 32, 64, "f32", "gelu"),
        # last layer, onto the SH coefficients that are there, a row for each pixel of the 1m workload's image
        _linear("layer-pixels-sh", "linear", 1237 * 822, 64, 48, "bf16", "none", residual=True),
        # a wide layer over a batch of tokens: bound by the matrix cores
        _linear("layer-wide", "linear", 4096, 1024, 4096, "f16", "gelu", residual=True),
        # gradient of the first layer over the small workload's Gaussians
        _linear("layer-grad-small", "linear_backward", 100_000, 32, 64, "f32", "gelu"),
        # gradient of a hidden layer over the 1m workload's Gaussians
        _linear("layer-grad-1m", "linear_backward", 1_000_000, 64, 128, "bf16", "silu"),
        # dropout on the SH rows of a cluster's Gaussians: a small call
        _dropout("dropout-small", 100, 48, "f32", 0.1, False),
        # dropout on the hidden activations of the 1m workload, added to the block's input
        _dropout("dropout-1m", 1_000_000, 128, "bf16", 0.1, True),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    do = rng.choice(["embedding", "embedding_backward", "linear", "linear", "linear_backward", "linear_backward",
                     "dropout"])
    dtype = rng.choice(["f32", "bf16", "f16"])
    pad = rng.choice([0, 0, 8, 3])
    size = 1 if dtype == "f32" else 2  # float32 cases have half the elements of the 16-bit ones
    if do.startswith("embedding"):
        n = _log(rng, 1, 1_048_576)
        dim = _log(rng, 1, min(1024, max(32_000_000 * size // n, 1)))
        vocab = _log(rng, 16, min(131_072, 32_000_000 * size // dim))
        c = _embedding("", do, n, dim, vocab, dtype, rng.choice(["int64", "int32"]), rng.choice([True, False]),
                       rng.choice([True, False]), pad)
    elif do == "dropout":
        rows = _log(rng, 1, 1_048_576)
        cols = _log(rng, 1, min(4096, max(60_000_000 * size // rows, 1)))
        c = _dropout("", rows, cols, dtype, rng.choice([0.1, 0.2, 0.5, 0.05]), rng.choice([True, False]), pad)
    else:
        rows = _log(rng, 1, 1_048_576)
        inputs = _log(rng, 1, min(4096, max(60_000_000 * size // rows, 1)))
        products = 2.0e9 if dtype == "f32" else 8.0e9
        outputs = _log(rng, 1, max(min(4096, 60_000_000 * size // rows, int(products / (rows * inputs))), 1))
        # a relu's derivative jumps at 0, where sums in another order fall on the other side: forward only
        act = rng.choice(["none", "silu", "gelu"] + (["relu"] if do == "linear" else []))
        c = _linear("", do, rows, inputs, outputs, dtype, act, rng.choice([True, True, False]),
                    do == "linear" and rng.choice([True, False]), pad)
    del c["name"]
    return c


# ---- inputs ----------------------------------------------------------------
def _rows(rows, cols, case, gen, scale=1.0):
    """[rows, cols] normal values; with "pad" a view of the first columns of a wider buffer."""
    t = torch.randn((rows, cols + case["pad"]), device="cuda", generator=gen) * scale
    return t.to(_TYPES[case["dtype"]])[:, :cols]


def _ids(case, gen):
    n, v = case["n"], case["vocab"]
    u = torch.rand(n, device="cuda", generator=gen, dtype=torch.float64)
    if case["skew"]:  # the r-th most frequent row is used about 1/r as often as the first
        order = torch.randperm(v, device="cuda", generator=gen)
        ids = order[((v + 1.0) ** u - 1.0).long().clamp_(0, v - 1)]
    else:
        ids = (u * v).long().clamp_(0, v - 1)
    if case["absent"]:  # Gaussians without a code
        ids = torch.where(torch.rand(n, device="cuda", generator=gen) < 0.02, -1, ids)
    return ids.to(torch.int32 if case["ids"] == "int32" else torch.int64)


def _inputs(case, seed):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(1_000_003 * int(seed) + 17)
    do = case["do"]
    if do == "embedding":
        return dict(table=_rows(case["vocab"], case["dim"], case, gen), ids=_ids(case, gen))
    if do == "embedding_backward":
        return dict(ids=_ids(case, gen), dl=_rows(case["n"], case["dim"], case, gen))
    if do == "dropout":
        x = _rows(case["rows"], case["cols"], case, gen)
        return dict(x=x, residual=_rows(case["rows"], case["cols"], case, gen) if case["residual"] else None,
                    seed=(0x9E3779B97F4A7C15 ^ (int(seed) * 0x1_0000_0001)) & (2 ** 64 - 1), offset=7 + int(seed) % 1000)
    m, k, n = case["rows"], case["inputs"], case["outputs"]
    s = dict(x=_rows(m, k, case, gen), weight=_rows(n, k, case, gen, k ** -0.5), bias=None)
    if case["bias"]:
        s["bias"] = (torch.randn(n, device="cuda", generator=gen) * 0.5).to(_TYPES[case["dtype"]])
    if do == "linear":
        s["residual"] = _rows(m, n, case, gen) if case["residual"] else None
    else:
        s["dl"] = _rows(m, n, case, gen)
    return s


def prepare(case, seed):
    s = _inputs(case, seed)
    s["case"] = case
    if own:  # a program keeps its output buffers and scratch from step to step
        from paper_2608_17298_amd import gart
        t = dict(device="cuda", dtype=_TYPES[case["dtype"]])
        do, nbytes = case["do"], 0
        if do == "embedding":
            s["out"] = torch.empty((case["n"], case["dim"]), **t)
        elif do == "embedding_backward":
            s["g_table"] = torch.empty((case["vocab"], case["dim"]), **t)
            nbytes = gart.gart_embedding_scratch_bytes(case["n"], case["vocab"], case["dim"])
        elif do == "dropout":
            s["y"] = torch.empty((case["rows"], case["cols"]), **t)
        else:
            m, k, n = case["rows"], case["inputs"], case["outputs"]
            if do == "linear":
                s["y"] = torch.empty((m, n), **t)
                nbytes = gart.gart_linear_scratch_bytes(m, k, n, t["dtype"])
            else:
                s["g_x"], s["g_weight"] = torch.empty((m, k), **t), torch.empty((n, k), **t)
                s["g_bias"] = torch.empty(n, **t) if case["bias"] else None
                nbytes = gart.gart_linear_backward_scratch_bytes(m, k, n, t["dtype"], case["act"])
        s["scratch"] = torch.empty(nbytes, dtype=torch.uint8, device="cuda")
        s["gart"] = gart
    return s


# ---- one pass --------------------------------------------------------------
_SCALE = 0.125  # of the looked-up rows
_GELU = math.sqrt(2.0 / math.pi)


def _own(s):
    case, g = s["case"], s["gart"]
    do = case["do"]
    if do == "embedding":
        g.gart_embedding(s["table"], s["ids"], s["out"], _SCALE)
        return s["out"]
    if do == "embedding_backward":
        g.gart_embedding_backward(s["ids"], s["dl"], s["g_table"], _SCALE, s["scratch"])
        return s["g_table"]
    if do == "dropout":
        g.gart_dropout(s["x"], s["y"], case["p"], s["seed"], s["offset"], s["residual"])
        return s["y"]
    if do == "linear":
        g.gart_linear(s["x"], s["weight"], s["y"], s["bias"], s["residual"], case["act"], s["scratch"])
        return s["y"]
    g.gart_linear_backward(s["x"], s["weight"], s["dl"], s["g_x"], s["g_weight"], s["g_bias"], s["bias"], case["act"],
                           s["scratch"])
    return [t for t in (s["g_x"], s["g_weight"], s["g_bias"]) if t is not None]


def _act(z, act):
    if act == "relu":
        return torch.clamp_min(z, 0.0)
    if act == "silu":
        return z / (1.0 + torch.exp(-z))
    if act == "gelu":
        return 0.5 * z * (1.0 + torch.tanh(_GELU * (z + 0.044715 * z * z * z)))
    return z


def _act_grad(z, act):
    if act == "silu":
        p = 1.0 / (1.0 + torch.exp(-z))
        return p * (1.0 + z * (1.0 - p))
    t = torch.tanh(_GELU * (z + 0.044715 * z * z * z))
    return 0.5 * (1.0 + t) + 0.5 * z * (1.0 - t * t) * _GELU * (1.0 + 0.134145 * z * z)


_M32 = 0xFFFFFFFF


def _philox(calls, offset, seed):
    """Four 32-bit words (in int64) of Philox-4x32-10 for the counters (calls, offset)."""
    c0, c1 = calls & _M32, calls >> 32
    c2, c3 = torch.full_like(calls, offset & _M32), torch.full_like(calls, offset >> 32)
    k0, k1 = seed & _M32, (seed >> 32) & _M32
    for _ in range(10):
        p0, p1 = c0 * 0xD2511F53, c2 * 0xCD9E8D57  # the low 64 bits of each product, in two's complement
        c0, c1, c2, c3 = ((p1 >> 32) & _M32) ^ c1 ^ k0, p1 & _M32, ((p0 >> 32) & _M32) ^ c3 ^ k1, p0 & _M32
        k0, k1 = (k0 + 0x9E3779B9) & _M32, (k1 + 0xBB67AE85) & _M32
    return c0, c1, c2, c3


def run(s):
    if own:
        return _own(s)
    case = s["case"]
    do, dt = case["do"], _TYPES[case["dtype"]]
    if do == "embedding":
        ids = s["ids"].long()
        ok = (ids >= 0) & (ids < case["vocab"])
        rows = s["table"][torch.where(ok, ids, 0)].float() * _SCALE
        return torch.where(ok[:, None], rows, 0.0).to(dt)
    if do == "embedding_backward":
        ids, v = s["ids"].long(), case["vocab"]
        ids = torch.where((ids >= 0) & (ids < v), ids, v)  # row v: what belongs to no entry
        g = torch.zeros((v + 1, case["dim"]), device="cuda")
        g.index_add_(0, ids, s["dl"].float())
        return (g[:v] * _SCALE).to(dt)
    if do == "dropout":
        x = s["x"].float()
        t = int(math.floor(case["p"] * 65536.0 + 0.5))
        calls = torch.arange((x.numel() + 7) // 8, device="cuda")
        words = _philox(calls, s["offset"], s["seed"])
        halves = torch.stack([h for w in words for h in (w & 0xFFFF, w >> 16)], dim=1)
        keep = (halves >= t).reshape(-1)[:x.numel()].reshape(x.shape)
        y = torch.where(keep, x * (65536.0 / (65536 - t)), 0.0)
        if s["residual"] is not None:
            y = y + s["residual"].float()
        return y.to(dt)
    x, w, act = s["x"].float(), s["weight"].float(), case["act"]
    if do == "linear":
        y = x @ w.t()
        if s["bias"] is not None:
            y = y + s["bias"].float()
        y = _act(y, act)
        if s["residual"] is not None:
            y = y + s["residual"].float()
        return y.to(dt)
    dz = s["dl"].float()
    if act != "none":
        z = x @ w.t()
        if s["bias"] is not None:
            z = z + s["bias"].float()
        dz = dz * _act_grad(z, act)
    out = [(dz @ w).to(dt), (dz.t() @ x).to(dt)]
    if s["bias"] is not None:
        out.append(dz.sum(0).to(dt))
    return out


# ---- what a pass cannot do without -------------------------------------------
def work(case):
    do, size = case["do"], 4 if case["dtype"] == "f32" else 2
    if do.startswith("embedding"):
        n, d, v = case["n"], case["dim"], case["vocab"]
        ids = n * (4 if case["ids"] == "int32" else 8)
        rows = min(n, v) if do == "embedding" else v  # table rows read, or gradient rows written
        return dict(bytes=ids + (n + rows) * d * size, flops=n * d)
    if do == "dropout":
        e = case["rows"] * case["cols"]
        return dict(bytes=e * size * (3 if case["residual"] else 2), flops=e * (2 if case["residual"] else 1))
    m, k, n = case["rows"], case["inputs"], case["outputs"]
    b = n if case["bias"] else 0
    if do == "linear":
        return dict(bytes=size * (m * k + n * k + b + m * n * (2 if case["residual"] else 1)), flops=2 * m * n * k)
    return dict(bytes=size * (2 * (m * k + n * k + b) + m * n), flops=(4 if case["act"] == "none" else 6) * m * n * k)


# ---- the definitions in 64 bits ------------------------------------------------
def _keep_exact(n, t, seed, offset):
    """The keep decisions of n elements, from the generator's definition."""
    out = np.empty(((n + 7) // 8, 8), dtype=bool)
    step = 1 << 17
    for a in range(0, len(out), step):
        i = np.arange(a, min(a + step, len(out)), dtype=np.uint64)
        ctr = [i & np.uint64(_M32), i >> np.uint64(32), np.full_like(i, offset & _M32), np.full_like(i, offset >> 32)]
        for r in range(10):
            ka = np.uint64((seed + r * 0x9E3779B9) & _M32)
            kb = np.uint64(((seed >> 32) + r * 0xBB67AE85) & _M32)
            pa, pb = ctr[0] * np.uint64(0xD2511F53), ctr[2] * np.uint64(0xCD9E8D57)
            ctr = [(pb >> np.uint64(32)) ^ ctr[1] ^ ka, pb & np.uint64(_M32), (pa >> np.uint64(32)) ^ ctr[3] ^ kb,
                   pa & np.uint64(_M32)]
        for j, word in enumerate(ctr):
            out[a:a + step, 2 * j] = (word & np.uint64(0xFFFF)) >= t
            out[a:a + step, 2 * j + 1] = (word >> np.uint64(16)) >= t
    return out.reshape(-1)[:n]


def exact(case, seed):
    s = _inputs(case, seed)
    do = case["do"]
    f64 = lambda t: t.cpu().to(torch.float64).numpy()  # noqa: E731
    if do == "embedding":
        table, ids = f64(s["table"]), s["ids"].cpu().numpy()
        out = np.zeros((case["n"], case["dim"]))
        has = np.flatnonzero((ids >= 0) & (ids < case["vocab"]))
        out[has] = table[ids[has]] * _SCALE
        return torch.from_numpy(out)
    if do == "embedding_backward":
        dl, ids = f64(s["dl"]), s["ids"].cpu().numpy()
        g = np.zeros((case["vocab"], case["dim"]))
        has = np.flatnonzero((ids >= 0) & (ids < case["vocab"]))
        has = has[np.argsort(ids[has], kind="stable")]
        if len(has):
            which, first = np.unique(ids[has], return_index=True)
            g[which] = np.add.reduceat(dl[has], first, axis=0) * _SCALE
        return torch.from_numpy(g)
    if do == "dropout":
        x = f64(s["x"])
        t = int(math.floor(case["p"] * 65536.0 + 0.5))
        keep = _keep_exact(x.size, t, s["seed"], s["offset"]).reshape(x.shape)
        x = np.where(keep, x * (65536.0 / (65536.0 - t)), 0.0)
        if s["residual"] is not None:
            x += f64(s["residual"])
        return torch.from_numpy(x)
    # products in 64 bits on the GPU
    x, w, act = s["x"].double(), s["weight"].double(), case["act"]
    b = x.new_zeros(case["outputs"]) if s["bias"] is None else s["bias"].double()
    z = torch.addmm(b, x, w.t().contiguous())
    u = z if act == "silu" else 2.0 * math.sqrt(2.0 / math.pi) * (z + 0.044715 * z ** 3)
    gate = torch.sigmoid(u)  # silu(z) = z gate(z), gelu(z) = z gate(2 sqrt(2 / pi) (z + 0.044715 z^3))
    if do == "linear":
        y = dict(none=z, relu=torch.where(z > 0, z, 0.0), silu=z * gate, gelu=z * gate)[act]
        return y if s["residual"] is None else y + s["residual"].double()
    du = 1.0 if act == "silu" else 2.0 * math.sqrt(2.0 / math.pi) * (1.0 + 3.0 * 0.044715 * z ** 2)
    dz = s["dl"].double() * (1.0 if act == "none" else gate + z * gate * torch.sigmoid(-u) * du)
    out = [torch.mm(dz, w), torch.mm(dz.t().contiguous(), x)]
    if s["bias"] is not None:
        out.append(dz.sum(dim=0))
    return out
