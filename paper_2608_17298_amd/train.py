"""Synthetic multi-view training step around the hot path.

One iteration on one view: gart_bounds -> gart_build_tile_map ->
gart_forward -> gart_l1_loss_grad (L1 against the view's target image) ->
gart_backward -> gart_adam_step per parameter group.  Every step runs in
the library's kernels; this module only orders the calls and owns the
device buffers (parameters are updated in place).

The paper trains with the 3DGS recipe (Adam over L1 plus SSIM for 30K
iterations); here the loss is the L1 sum alone, whose gradient sign(C - C*)
is the upstream gradient used throughout, and each parameter group has its
own Adam learning rate (3DGS-style defaults below).

With an appearance model (appearance.Appearance) the step renders the SH
coefficients that the model gives for the view, and its weights and the
view's codes are updated along with the scene: by Adam, or, with
appearance_optimizer="muon", its weight matrices by orthogonalised momentum
(gart_muon_step) and the rest by Adam.
"""
from __future__ import annotations

import dataclasses

import torch

from . import gart

# Per-group Adam learning rates (3DGS-style defaults; SH bands share one rate).
DEFAULT_LR = dict(means=1.6e-4, log_scales=5e-3, quats=1e-3, logits=5e-2, sh=2.5e-3)
APPEARANCE_LR = 1e-3  # weights and codes of an appearance model
# Of the matrices' orthogonalised steps: the publication's polynomial and rates.
MUON_LR, MUON_MOMENTUM = 0.02, 0.95
NEWTON_SCHULZ = (3.4445, -4.7750, 2.0315, 1e-7, 5)
GROUPS = ("means", "log_scales", "quats", "logits", "sh")
_PARAM_ATTR = dict(means="means", log_scales="log_scales", quats="quats", logits="opacity_logits", sh="sh")


class Trainer:
    """Adam on the Gaussians of `scene` over a set of views with target images."""

    def __init__(self, scene, cameras, targets, tile=None, mode="gather", lr=None, betas=(0.9, 0.999),
                 eps=1e-15, stream=None, appearance=None, appearance_lr=APPEARANCE_LR, appearance_optimizer="adam",
                 muon_lr=MUON_LR, muon_decay=0.0):
        if len(cameras) != len(targets) or not cameras:
            raise ValueError("one target image per camera")
        self.g = gart.Gaussians.from_scene(scene)
        self.settings = gart.make_settings(tile or scene.tile, mode)
        self.cams = [gart.make_camera(c) for c in cameras]
        w, h = self.cams[0].width, self.cams[0].height
        if any(c.width != w or c.height != h for c in self.cams):
            raise ValueError("views must share one image size")
        self.targets = [t.contiguous() for t in targets]
        self.stream = stream
        self.frame = None
        dev = self.g.means.device
        self.image = torch.empty((h, w, 3), dtype=torch.float32, device=dev)
        self.dl = torch.empty_like(self.image)
        self.loss = torch.zeros(1, dtype=torch.float64, device=dev)
        self.partial = torch.empty(gart.gart_l1_partials(self.image.numel()), dtype=torch.float64, device=dev)
        self.grads = gart.empty_grads(self.g)
        lr = dict(DEFAULT_LR, **(lr or {}))
        self.adam = {k: gart.gart_adam(lr[k], betas[0], betas[1], eps) for k in GROUPS}
        self.m = {k: torch.zeros_like(self.param(k)) for k in GROUPS}
        self.v = {k: torch.zeros_like(self.param(k)) for k in GROUPS}
        self.t = 0
        self.appearance = appearance
        if appearance_optimizer not in ("adam", "muon"):
            raise ValueError(f"unknown optimizer {appearance_optimizer!r}")
        if appearance is not None:
            if appearance.codes.shape[0] != self.g.n or appearance.table.shape[0] < len(cameras):
                raise ValueError("the appearance model is not of this scene's Gaussians and views")
            self.appearance_adam = gart.gart_adam(appearance_lr, betas[0], betas[1], eps)
            # moments of the weights, and of each view's codes, which step only when the view is used
            self.am, self.av = ({k: torch.zeros_like(appearance.params[k]) for k in appearance.names} for _ in range(2))
            self.tm, self.tv = torch.zeros_like(appearance.table), torch.zeros_like(appearance.table)
            self.view_t = [0] * len(cameras)
            self.muon = {}  # of the matrices that it steps; am is their momentum
            if appearance_optimizer == "muon":
                how, need = gart.gart_newton_schulz(*NEWTON_SCHULZ), 0
                for k in appearance.names:
                    if appearance.params[k].dim() == 2:
                        rows, cols = appearance.params[k].shape
                        scale = max(1.0, rows / cols) ** 0.5  # rows of a tall update are as large as a square one's
                        self.muon[k] = gart.gart_muon(muon_lr, MUON_MOMENTUM, muon_decay, scale, 1, how)
                        need = max(need, gart.gart_muon_scratch_bytes(rows, cols))
                        del self.av[k]
                self.muon_scratch = torch.empty(need, dtype=torch.uint8, device=dev)

    def param(self, k):
        return getattr(self.g, _PARAM_ATTR[k])

    def _appearance_step(self, view):
        """Gradients of the appearance model from that of the SH coefficients, and its steps."""
        a, h, s = self.appearance, self.appearance_adam, self.stream
        a.backward(self.grads["sh"], self.t, stream=s)
        for k in a.names:
            if k in self.muon:
                gart.gart_muon_step(a.params[k], a.grads[k], self.am[k], self.muon[k], self.muon_scratch, stream=s)
                continue
            gart.gart_adam_step(a.params[k], a.grads[k], self.am[k], self.av[k], h, self.t, stream=s)
        self.view_t[view] += 1
        gart.gart_adam_step(a.table[view], a.g_table, self.tm[view], self.tv[view], h, self.view_t[view], stream=s)

    def step(self, view: int, events=None):
        """One iteration on view `view`; returns the device fp64 loss.  With
        `events` (6 torch.cuda.Event), records them between the stages."""
        cam, s = self.cams[view], self.stream

        def mark(k):
            if events is not None:
                events[k].record(torch.cuda.current_stream() if s is None else s)

        mark(0)
        g = self.g
        if self.appearance is not None:  # the step's number is t + 1, there and in the gradient
            g = dataclasses.replace(g, sh=self.appearance.forward(view, g.sh, self.t + 1, stream=s))
        self.frame = gart.prepare(g, cam, self.settings, self.frame, stream=s)
        mark(1)
        gart.gart_forward(g, cam, self.settings, self.frame, self.image, stream=s)
        mark(2)
        gart.gart_l1_loss_grad(self.image, self.targets[view], self.dl, self.loss, self.partial, stream=s)
        mark(3)
        gart.gart_backward(g, cam, self.settings, self.frame, self.dl, self.grads, stream=s)
        mark(4)
        self.t += 1
        if self.appearance is not None:
            self._appearance_step(view)
        for k in GROUPS:
            gart.gart_adam_step(self.param(k), self.grads[k], self.m[k], self.v[k], self.adam[k], self.t, stream=s)
        mark(5)
        return self.loss
