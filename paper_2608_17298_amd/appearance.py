"""Appearance model: the SH coefficients of every Gaussian, corrected per view by a learned function of a code.

Captures whose light, exposure or weather change from view to view cannot be fitted by one set of colours.  Every
Gaussian names a code (a cluster of Gaussians shares one; -1: none), each view has its own row for each code, and

    e  = scale * table[view][code]              gart_embedding
    n  = layer norm of e, gain and shift        gart_layer_norm (norm=True; else n = e)
    h  = act(n w1^T + b1)                       gart_linear
    d  = dropout(h)                             gart_dropout, mask of (seed, step), never stored
    sh = sh_base + d w2^T + b2                  gart_linear, residual

sh takes the place of the scene's SH coefficients in gart_bounds, gart_forward and gart_backward, and the gradient of
sh goes back through the block: to the weights, to the view's rows of the table, and unchanged to sh_base.  w2 and b2
start at zero, so training starts from the scene as it is.  With the norm, codes of any size meet w1 alike; a
Gaussian without a code has a row of zeros, whose norm is the shift.
"""
from __future__ import annotations

import torch

from . import gart

NORM_EPS = 1e-5


class Appearance:
    """The block's parameters, buffers and gradients for `codes` (int32 or int64 [N], values below n_codes)."""

    def __init__(self, codes: torch.Tensor, n_codes: int, n_views: int, sh_cols: int, width: int = 32,
                 hidden: int = 64, act: str = "gelu", dropout: float = 0.1, scale: float = 1.0, seed: int = 0,
                 norm: bool = False):
        if codes.dim() != 1 or codes.dtype not in (torch.int32, torch.int64):
            raise ValueError("codes must be a 1-D int32 or int64 tensor")
        self.codes, self.act, self.p, self.scale = codes.contiguous(), act, float(dropout), float(scale)
        self.seed, self.norm = int(seed), bool(norm)
        n, dev = codes.shape[0], codes.device
        gen = torch.Generator().manual_seed(self.seed)
        uniform = lambda *s, k: ((torch.rand(s, generator=gen) * 2.0 - 1.0) * k ** -0.5).to(dev)  # noqa: E731
        self.table = (torch.randn((n_views, n_codes, width), generator=gen) * 0.1).to(dev)
        self.params = dict(w1=uniform(hidden, width, k=width), b1=uniform(hidden, k=width),
                           w2=torch.zeros((sh_cols, hidden), device=dev), b2=torch.zeros(sh_cols, device=dev))
        if self.norm:
            self.params.update(gain=torch.ones(width, device=dev), shift=torch.zeros(width, device=dev))
        self.names = tuple(self.params)  # of what a step updates, besides the table
        self.grads = {k: torch.zeros_like(v) for k, v in self.params.items()}
        self.g_table = torch.zeros((n_codes, width), device=dev)  # of the rows of the view last used
        f = dict(dtype=torch.float32, device=dev)
        self.e, self.g_e = torch.empty((n, width), **f), torch.empty((n, width), **f)
        self.n, self.g_n = (torch.empty((n, width), **f) for _ in range(2)) if self.norm else (self.e, self.g_e)
        self.h, self.d, self.g_d = (torch.empty((n, hidden), **f) for _ in range(3))
        self.sh = torch.empty((n, sh_cols), **f)
        need = max(gart.gart_linear_scratch_bytes(n, width, hidden), gart.gart_linear_scratch_bytes(n, hidden, sh_cols),
                   gart.gart_linear_backward_scratch_bytes(n, width, hidden, act=act),
                   gart.gart_linear_backward_scratch_bytes(n, hidden, sh_cols),
                   gart.gart_embedding_scratch_bytes(n, n_codes, width),
                   gart.gart_layer_norm_backward_scratch_bytes(n, width) if self.norm else 0)
        self.scratch = torch.empty(need, dtype=torch.uint8, device=dev)

    def forward(self, view: int, sh_base: torch.Tensor, step: int = 0, train: bool = True, stream=None) -> torch.Tensor:
        """SH coefficients for `view`, shaped like sh_base [N, K, 3].  In training, the dropout's mask is that of
        `step`; otherwise nothing is dropped."""
        p, n = self.params, self.codes.shape[0]
        gart.gart_embedding(self.table[view], self.codes, self.e, self.scale, stream=stream)
        if self.norm:
            gart.gart_layer_norm(self.e, self.n, p["gain"], p["shift"], NORM_EPS, stream=stream)
        gart.gart_linear(self.n, p["w1"], self.h, p["b1"], None, self.act, self.scratch, stream=stream)
        gart.gart_dropout(self.h, self.d, self.p if train else 0.0, self.seed, step, stream=stream)
        gart.gart_linear(self.d, p["w2"], self.sh, p["b2"], sh_base.view(n, self.sh.shape[1]), "none", self.scratch,
                         stream=stream)
        return self.sh.view(sh_base.shape)

    def backward(self, g_sh: torch.Tensor, step: int = 0, stream=None):
        """Gradients (self.grads, self.g_table) of the training forward that ran last, with the same step, from that
        of its SH coefficients, which is also sh_base's."""
        p, g, n = self.params, self.grads, self.codes.shape[0]
        gart.gart_linear_backward(self.d, p["w2"], g_sh.view(n, self.sh.shape[1]), self.g_d, g["w2"], g["b2"], p["b2"],
                                  "none", self.scratch, stream=stream)
        gart.gart_dropout(self.g_d, self.g_d, self.p, self.seed, step, stream=stream)
        gart.gart_linear_backward(self.n, p["w1"], self.g_d, self.g_n, g["w1"], g["b1"], p["b1"], self.act,
                                  self.scratch, stream=stream)
        if self.norm:
            gart.gart_layer_norm_backward(self.e, self.g_n, self.g_e, g["gain"], g["shift"], p["gain"], NORM_EPS,
                                          self.scratch, stream=stream)
        gart.gart_embedding_backward(self.codes, self.g_e, self.g_table, self.scale, self.scratch, stream=stream)
