"""Plain 64-bit forms of the learned blocks (embedding, linear layer, dropout), with numpy, and the bounds on the
kernels' errors that their arithmetic implies."""
import math

import numpy as np

U32 = 2.0 ** -24
U = dict(f32=2.0 ** -24, bf16=2.0 ** -8, f16=2.0 ** -11)      # largest relative error of a rounding to the type
TINY = dict(f32=2.0 ** -126, bf16=2.0 ** -126, f16=2.0 ** -24)  # rounding near zero (subnormals)


def embedding(table, ids, scale):
    out = np.zeros((len(ids), table.shape[1]))
    for i, v in enumerate(ids):
        if 0 <= v < len(table):
            out[i] = scale * table[v]
    return out


def embedding_grad(ids, dl, vocab, scale):
    """The gradient and, for its error bound, the sums of absolute values times the number of terms."""
    g, a, c = np.zeros((vocab, dl.shape[1])), np.zeros((vocab, dl.shape[1])), np.zeros((vocab, 1))
    ok = (ids >= 0) & (ids < vocab)
    np.add.at(g, ids[ok], dl[ok])
    np.add.at(a, ids[ok], np.abs(dl[ok]))
    np.add.at(c[:, 0], ids[ok], 1.0)
    return scale * g, abs(scale) * a * (c + 2.0)


def act(z, name):
    if name == "relu":
        return np.maximum(z, 0.0)
    if name == "silu":
        return z / (1.0 + np.exp(-z))
    if name == "gelu":
        return 0.5 * z * (1.0 + np.tanh(math.sqrt(2.0 / math.pi) * (z + 0.044715 * z ** 3)))
    return z


def act_grad(z, name):
    if name == "relu":
        return (z > 0).astype(np.float64)
    if name == "silu":
        s = 1.0 / (1.0 + np.exp(-z))
        return s + z * s * (1.0 - s)
    if name == "gelu":
        c = math.sqrt(2.0 / math.pi)
        t = np.tanh(c * (z + 0.044715 * z ** 3))
        return 0.5 * (1.0 + t) + 0.5 * z * (1.0 - t * t) * c * (1.0 + 3 * 0.044715 * z * z)
    return np.ones_like(z)


def linear(x, w, bias, residual, name):
    z = x @ w.T + (0.0 if bias is None else bias)
    return act(z, name) + (0.0 if residual is None else residual)


def linear_tolerance(x, w, bias, residual, name, dtype):
    """Sums of k float products in any order are off by at most about k u sum|x||w|; |act'| <= 1.13; an activation's
    own arithmetic (an exponential of a rounded argument, a reciprocal) by a few u of |z| (1 + |z|)."""
    k = x.shape[1]
    a = np.abs(x) @ np.abs(w).T + (0.0 if bias is None else np.abs(bias))
    z = x @ w.T + (0.0 if bias is None else bias)
    r = 0.0 if residual is None else np.abs(residual)
    y = linear(x, w, bias, residual, name)
    own = 0.0 if name in ("none", "relu") else 8.0 * U32 * np.abs(z) * (1.0 + np.abs(z))
    return 1.01 * U[dtype] * np.abs(y) + U32 * (1.2 * (k + 4) * a + 2.0 * (np.abs(z) + r)) + own + TINY[dtype]


def linear_grads(x, w, bias, dl, name):
    z = x @ w.T + (0.0 if bias is None else bias)
    dz = dl * act_grad(z, name)
    return dz @ w, dz.T @ x, dz.sum(axis=0)


def linear_grads_tolerance(x, w, bias, dl, name, dtype):
    """dz is off by the slope's error (|act''| <= 1.2 times z's, and the activation's own arithmetic) and, where it is
    stored in 16 bits for the products, by one rounding; sums as in linear_tolerance."""
    m, k = x.shape
    n = w.shape[0]
    z = x @ w.T + (0.0 if bias is None else bias)
    a = np.abs(x) @ np.abs(w).T + (0.0 if bias is None else np.abs(bias))
    dz = dl * act_grad(z, name)
    e = np.zeros_like(dz)
    if name in ("silu", "gelu"):
        e = np.abs(dl) * U32 * (1.2 * (k + 4) * a + 16.0 * (1.0 + np.abs(z)) ** 2)
    er = e + (0.0 if name == "none" else 1.01 * U[dtype] * np.abs(dz) + TINY[dtype])
    gx, gw, gb = linear_grads(x, w, bias, dl, name)

    def one(g, terms, size, err):
        return 1.01 * U[dtype] * np.abs(g) + 1.2 * U32 * (terms + 4) * size + err + TINY[dtype]

    ax, aw, ad = np.abs(x), np.abs(w), np.abs(dz) + er
    return (one(gx, n, ad @ aw, er @ aw), one(gw, m, ad.T @ ax, er.T @ ax),
            one(gb, m, (np.abs(dz) + e).sum(axis=0), e.sum(axis=0)))


def philox(call, offset, seed):
    """Philox-4x32-10 of Salmon, Moraes, Dror and Shaw (2011) with Python integers."""
    m32 = 0xFFFFFFFF
    c = [call & m32, call >> 32, offset & m32, offset >> 32]
    k = [seed & m32, seed >> 32]
    for _ in range(10):
        p0, p1 = 0xD2511F53 * c[0], 0xCD9E8D57 * c[2]
        c = [(p1 >> 32) ^ c[1] ^ k[0], p1 & m32, (p0 >> 32) ^ c[3] ^ k[1], p0 & m32]
        k = [(k[0] + 0x9E3779B9) & m32, (k[1] + 0xBB67AE85) & m32]
    return c


def keep(n, p, seed, offset, first=0):
    """Keep decisions of elements first .. first + n - 1."""
    t = int(math.floor(float(np.float32(p)) * 65536.0 + 0.5))
    out, words, call = np.empty(n, dtype=bool), None, -1
    for i in range(n):
        e = first + i
        if e // 8 != call:
            call = e // 8
            words = philox(call, offset, seed)
        out[i] = (words[e % 8 // 2] >> (16 * (e % 2))) & 0xFFFF >= t
    return out


def dropout(x, residual, p, seed, offset):
    t = int(math.floor(float(np.float32(p)) * 65536.0 + 0.5))
    s = 65536.0 / (65536.0 - t) if t < 65536 else 0.0
    k = keep(x.size, p, seed, offset).reshape(x.shape)
    return np.where(k, x * s, 0.0) + (0.0 if residual is None else residual)


def dropout_tolerance(x, residual, p, dtype, y):
    s = 1.0 / (1.0 - p) if p < 1 else 0.0
    return 1.01 * U[dtype] * np.abs(y) + 4.0 * U32 * (np.abs(x) * s + (0.0 if residual is None else np.abs(residual))) \
        + TINY[dtype]
