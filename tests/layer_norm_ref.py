"""Plain 64-bit forms of the layer norm and its gradient, with numpy, and the bounds on the kernels' errors that their
arithmetic implies."""
import numpy as np

from blocks_ref import TINY, U, U32


def _steps(cols):
    """Additions that any element of a row's sum passes: a lane adds up to 64 elements of its own, or one in 1024
    packs of a long row (fewer than cols / 256), and lanes and waves are joined in at most 16 more."""
    return 80 + cols / 256


def _stats(x, eps):
    d = x - x.mean(axis=1, keepdims=True)
    var = (d * d).mean(axis=1, keepdims=True)
    return d, var, 1.0 / np.sqrt(var + eps)


def norm(x, gain, bias, eps):
    d, _, rstd = _stats(x, eps)
    h = d * rstd * (1.0 if gain is None else gain)
    return h + (0.0 if bias is None else bias)


def _errors(x, eps):
    """d and rstd, and bounds on their errors: of the mean's sum, of each difference, of the sum of squares, and two
    units of the last place for the square root's reciprocal."""
    n = _steps(x.shape[1])
    d, var, rstd = _stats(x, eps)
    e_mean = n * U32 * np.abs(x).mean(axis=1, keepdims=True)
    e_d = e_mean + U32 * np.abs(d)
    e_var = (n + 3) * U32 * var + 2.0 * (np.abs(d) * e_d).mean(axis=1, keepdims=True) + (e_d ** 2).mean(axis=1, keepdims=True)
    e_rstd = rstd * (0.5 * e_var / (var + eps) + 6.0 * U32)
    return d, rstd, 1.05 * e_d, 1.05 * e_rstd


def norm_tolerance(x, gain, bias, eps, dtype):
    d, rstd, e_d, e_rstd = _errors(x, eps)
    g = 1.0 if gain is None else np.abs(gain)
    y = norm(x, gain, bias, eps)
    h = np.abs(d) * rstd * g
    own = U32 * (3.0 * h + np.abs(y))
    return 1.01 * U[dtype] * np.abs(y) + 1.05 * (g * (rstd * e_d + np.abs(d) * e_rstd) + own) + TINY[dtype]


def norm_grads(x, dl, gain, eps):
    d, _, rstd = _stats(x, eps)
    h = d * rstd
    w = dl if gain is None else dl * gain
    g_x = rstd * (w - w.mean(axis=1, keepdims=True) - h * (w * h).mean(axis=1, keepdims=True))
    return g_x, (dl * h).sum(axis=0), dl.sum(axis=0)


def norm_grads_tolerance(x, dl, gain, eps, dtype):
    """As above, with the sums of w and w h of as many steps; sums over the rows of one step a row at most."""
    n, rows = _steps(x.shape[1]), x.shape[0]
    d, rstd, e_d, e_rstd = _errors(x, eps)
    w = np.abs(dl if gain is None else dl * gain)
    mean = lambda v: v.mean(axis=1, keepdims=True)  # noqa: E731
    h, e_h = np.abs(d) * rstd, rstd * e_d + np.abs(d) * e_rstd
    along = mean(w * h)
    e_mw = (n + 2) * U32 * mean(w)
    e_along = (n + 6) * U32 * along + mean(w * e_h)
    e_in = U32 * (4.0 * w + 2.0 * mean(w) + 5.0 * h * along) + e_mw + h * e_along + e_h * along
    g_x, g_gain, g_bias = norm_grads(x, dl, gain, eps)
    inner = w + mean(w) + h * along
    gx = 1.01 * U[dtype] * np.abs(g_x) + 1.1 * (rstd * e_in + e_rstd * inner) + TINY[dtype]
    a = np.abs(dl)
    gg = 1.01 * U[dtype] * np.abs(g_gain) + 1.1 * ((rows + 4) * U32 * (a * (h + e_h)).sum(axis=0) + (a * e_h).sum(axis=0))
    gb = 1.01 * U[dtype] * np.abs(g_bias) + 1.1 * (rows + 2) * U32 * a.sum(axis=0)
    return gx, gg + TINY[dtype], gb + TINY[dtype]
