"""Plain forms of the orthogonalising iteration and of the momentum step that uses it, with numpy in 64 bits and, as a
yardstick of what float32 can reach, in 32; and bounds on the kernels' errors that their arithmetic implies."""
import numpy as np

from blocks_ref import U, U32

COEFFICIENTS = (3.4445, -4.7750, 2.0315)
EPS = 1e-7


def coefficients():
    """As the call takes them: float32."""
    return [float(np.float32(v)) for v in COEFFICIENTS]


def orthogonalize(x, steps=5, abc=None, eps=EPS, dtype=np.float64):
    a, b, c = (dtype(v) for v in (abc or coefficients()))
    norm = np.sqrt((x.astype(np.float64) ** 2).sum()) + float(np.float32(eps))
    x = (x / norm).astype(dtype)
    flat = x if x.shape[0] <= x.shape[1] else x.T
    for _ in range(steps):
        q = flat @ flat.T
        flat = a * flat + (b * q + c * (q @ q)) @ flat
    return flat if x.shape[0] <= x.shape[1] else flat.T


def singular_values(s, steps=5, abc=None):
    a, b, c = abc or coefficients()
    for _ in range(steps):
        s = a * s + b * s ** 3 + c * s ** 5
    return s


def one_step_tolerance(x, dtype, abc=None, eps=EPS):
    """One step, element by element.  Operands have 22 bits (2^-22 of the element, and 2^-38 of the bound on all of
    them) and their low parts' product is left out (2^-22): 12 u of a product's terms.  A sum of three products of k
    terms is off by about 3 k u of its terms."""
    a, b, c = abc or coefficients()
    norm = np.sqrt((x ** 2).sum()) + float(np.float32(eps))
    x = x / norm
    tall = x.shape[0] > x.shape[1]
    if tall:
        x = x.T
    n, m = x.shape
    ax, floor = np.abs(x), 2.0 ** -38
    e0 = 8 * U32 * ax + floor
    q = x @ x.T
    aq = np.abs(q)
    eq = 1.2 * U32 * (3 * m + 16) * (ax @ ax.T) + e0 @ ax.T + ax @ e0.T + 4 * U32 * aq + floor
    p = b * q + c * (q @ q)
    ap, size = np.abs(p), abs(b) * aq + abs(c) * (aq @ aq)
    ep = abs(b) * eq + abs(c) * (aq @ eq + eq @ aq + 1.2 * U32 * (3 * n + 16) * (aq @ aq)) + 8 * U32 * size \
        + floor * (abs(b) + abs(c))
    y = a * x + p @ x
    e = abs(a) * e0 + ep @ ax + ap @ e0 + 1.2 * U32 * (3 * n + 16) * (ap @ ax) + 4 * U32 * (abs(a) * ax + ap @ ax)
    t = 1.05 * e + 1.01 * U[dtype] * np.abs(y) + U[dtype] * 2.0 ** -13
    return t.T if tall else t


def muon(param, grad, m, lr, momentum, decay, scale, nesterov, steps=5, dtype=np.float64):
    f = lambda v: float(np.float32(v))  # noqa: E731
    mu = dtype(f(momentum))
    m = (mu * m.astype(dtype) + grad.astype(dtype)).astype(dtype)
    u = grad.astype(dtype) + mu * m if nesterov else m
    o = orthogonalize(u, steps, dtype=dtype)
    p = param.astype(dtype)
    return p - dtype(f(lr) * f(decay)) * p - dtype(f(lr) * f(scale)) * o, m, o
