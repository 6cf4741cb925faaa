"""The attention block around the cached attention: what makes its queries and takes its output.

Per layer, for a batch whose rows belong to different agents (``agent_id``; -1: the adapter-free view):

    r  = r + y                        the residual stream takes the previous layer's output        ) one call,
    h  = norm(r) * gain               hidden states; with ``e4m3`` also in 8 bits with a scale a row ) ``rms_norm``
    q  = h W_q + s (h A_q) B_q        ``adapted_project`` (8 bits: ``adapted_project_e4m3``)
    ... the caller projects h into its caches and attends with q ...
    y  = o W_o + s (o A_o) B_o        ``adapted_project``

Adapters sit on the query and output projections with the rank of the value side (none where that is 0); the cached keys and values
have theirs in the layer itself.  The paper adapts Q and V by default (Section 2.1); which projections carry adapters is the caller's choice.
"""
from __future__ import annotations

from typing import Callable, Optional

import torch

from . import inputs as I
from .binding import Precc

EPS = 1e-5


class AttentionBlocks:
    """Weights, residual stream and scratch of a stack of layers (distinct weights per layer unless ``shared_weights``)."""

    def __init__(self, px: Precc, geo: I.Geometry, n_layers: int, max_rows: int, seed: int = 0, shared_weights: bool = False, e4m3: bool = False):
        if n_layers < 1 or max_rows < 1:
            raise ValueError("a stack of blocks has at least one layer and one row")
        self.px, self.geo, self.n_layers, self.e4m3 = px, geo, n_layers, e4m3
        d, width = geo.d_model, geo.n_q * geo.hd
        scale = geo.scale(geo.rank_v)
        self.W_q, self.W_o, self.gain = [], [], []
        for l in range(1 if shared_weights else n_layers):
            w = {k: v.cuda() for k, v in I.block_weights(geo, seed, f"L{l}").items()}
            lora = geo.rank_v > 0
            self.W_q.append(px.adapted_weights(w["W_q"], w["A_q"] if lora else None, w["B_q"] if lora else None, scale, e4m3=e4m3))
            self.W_o.append(px.adapted_weights(w["W_o"], w["A_o"] if lora else None, w["B_o"] if lora else None, scale))
            self.gain.append(w["gain"])

        def mk(cols, dtype=torch.bfloat16):
            return torch.empty((max_rows, cols), dtype=dtype, device="cuda")
        self.r, self.h, self.y, self.q, self.o = mk(d), mk(d), mk(d), mk(width), mk(width)
        self.h8 = mk(d, torch.float8_e4m3fn) if e4m3 else None
        self.h_scale = torch.empty(max_rows, dtype=torch.float32, device="cuda") if e4m3 else None
        self.ws = px.adapted_workspace(self.W_q[0], max_rows)          # (both projections have the same rank, and run one after the other)

    def forward(self, x: torch.Tensor, agent_id: Optional[torch.Tensor], attend: Callable[[int, torch.Tensor, torch.Tensor, torch.Tensor], None]) -> torch.Tensor:
        """Rows x [n, d_model] of the residual stream through all layers.  ``attend(layer, h, q, out)`` writes h [n, d_model] into the
        layer's caches and the attention of q [n, n_q, hd] into out.  Returns the residual stream after the last layer (a buffer
        of this object, overwritten by the next call)."""
        n, px, geo = x.shape[0], self.px, self.geo
        if n > self.r.shape[0] or x.shape[1:] != self.r.shape[1:]:
            raise ValueError(f"x is {tuple(x.shape)}, the blocks take up to {self.r.shape[0]} rows of {self.r.shape[1]}")
        r, h, y, q, o = (t[:n] for t in (self.r, self.h, self.y, self.q, self.o))
        h8, hs = (self.h8[:n], self.h_scale[:n]) if self.e4m3 else (None, None)
        r.copy_(x)
        for l in range(self.n_layers):
            k = l % len(self.W_q)
            if l == 0:
                px.rms_norm(r, self.gain[k], EPS, out=h, out_e4m3=h8, out_scale=hs)
            else:
                px.rms_norm(y, self.gain[k], EPS, out=h, residual=r, residual_out=r, out_e4m3=h8, out_scale=hs)
            if self.e4m3:
                px.adapted_project_e4m3(self.W_q[k], h8, hs, q, agent_id, self.ws)
            else:
                px.adapted_project(self.W_q[k], h, q, agent_id, self.ws)
            attend(l, h, q.view(n, geo.n_q, geo.hd), o.view(n, geo.n_q, geo.hd))
            px.adapted_project(self.W_o[k], o, y, agent_id, self.ws)
        px.rms_norm(y, self.gain[0], EPS, out=h, residual=r, residual_out=r)
        return r
