"""What may stand between a last stage's layers and its output projection: a final norm, and in front of it a residual projection in
microscaled 8- or 4-bit floating point whose result is dropped out in training.

    without projection:  n = rmsnorm(y; g_norm)
    with it:             b = Q(rmsnorm(y; g_proj)) Q(W)^T,   h = y + dropout(b),   n = rmsnorm(h; g_norm)

``Tail`` holds the parameters, their fp32 gradients and one micro-batch's activations.  Gradients pass a packed operand as if it were the tensor
that was packed:  with d the gradient of b,  d(rmsnorm(y)) = Q(d) Q(W^T)^T  and  dW += Q(d^T) Q(rmsnorm(y)^T)^T, each operand packed
along the axis that is summed over.
"""
from __future__ import annotations

import numpy as np
import torch

from . import binding as hh
from . import glue as L

FORMATS = {"e4m3": hh.HH_MX_E4M3, "e2m1": hh.HH_MX_E2M1}


class Packed:
    """Buffers of a packed tensor."""

    def __init__(self, rows: int, k: int, format: int):
        c, s = hh.hh_mx_sizes(format, rows, k)
        self.buffers = torch.empty(c, dtype=torch.uint8, device=L.DEV), torch.empty(s, dtype=torch.uint8, device=L.DEV)
        self.struct = hh.make_mx(*self.buffers)


class Tail:
    """``g_norm``: [hidden]; ``g_proj`` [hidden] and ``w_proj`` [hidden, hidden]: None without the projection."""

    def __init__(self, tokens: int, hidden: int, bf16: bool, g_norm: np.ndarray, g_proj: np.ndarray | None = None, w_proj: np.ndarray | None = None,
                 format: str = "e4m3", dropout: float = 0.0, seed: int = 0, eps: float = 1e-5):
        if (g_proj is None) != (w_proj is None) or (dropout and w_proj is None):
            raise ValueError("a projection has a gain and a weight, and dropout needs one")
        self.tokens, self.hidden, self.dropout, self.seed, self.projects = tokens, hidden, dropout, seed, w_proj is not None
        self.dtype = hh.HH_BF16 if bf16 else hh.HH_F32
        dt = torch.bfloat16 if bf16 else torch.float32
        self.w = {"g_norm": L.to_dev(g_norm, bf16)}
        if self.projects:
            self.w.update(g_proj=L.to_dev(g_proj, bf16), w_proj=L.to_dev(w_proj, bf16))
        self.g = {n: torch.zeros(t.shape, dtype=torch.float32, device=L.DEV) for n, t in self.w.items()}
        self.normed = torch.empty(tokens, hidden, dtype=dt, device=L.DEV)
        self.norm_cfg = hh.make_add_norm_cfg(tokens, hidden, eps, self.dtype)
        self.workspace_bytes = hh.hh_add_norm_sizes(self.norm_cfg)
        if not self.projects:
            return
        self.format = f = FORMATS[format]
        self.proj_cfg = hh.make_add_norm_cfg(tokens, hidden, eps, self.dtype, f)
        # of the input's gradient too.  Fast sums: their error of 2^-16 of a result is a 4000th of what packing the operands leaves (E4M3, 2^-4 a value)
        self.fwd_cfg = hh.make_mx_product_cfg(tokens, hidden, hidden, f, f, self.dtype, sums=hh.HH_MX_SUMS_FAST)
        self.weight_cfg = hh.make_mx_product_cfg(hidden, hidden, tokens, f, f, hh.HH_F32)
        self.workspace_bytes = max(self.workspace_bytes, hh.hh_mx_product_sizes(self.fwd_cfg), hh.hh_mx_product_sizes(self.weight_cfg))
        self.x, self.branch, self.sum, self.dbranch, self.dx = (torch.empty_like(self.normed) for _ in range(5))
        self.q = {n: Packed(rows, k, f) for n, rows, k in (("x", tokens, hidden), ("x_t", hidden, tokens), ("w", hidden, hidden), ("w_t", hidden, hidden),
                                                           ("d", tokens, hidden), ("d_t", hidden, tokens))}

    def pack(self, ctx, stream) -> None:
        """The weight's packed copies: once after each update."""
        if self.projects:
            hh.hh_mx_quantise(ctx, self.hidden, self.hidden, self.dtype, self.w["w_proj"], self.hidden, self.format, self.q["w"].struct,
                              self.q["w_t"].struct, stream)

    def _drop(self, use: int):
        return hh.make_dropout(self.dropout, self.seed, use) if self.dropout else None

    def forward(self, ctx, y, use: int, ws, stream):
        """-> n [tokens, hidden] of y.  use: number of this pass, which names the values that are dropped; backward has the same."""
        if not self.projects:
            hh.hh_add_norm_fwd(ctx, self.norm_cfg, None, y, None, self.w["g_norm"], None, self.normed, None, stream)
            return self.normed
        hh.hh_add_norm_fwd(ctx, self.proj_cfg, None, y, None, self.w["g_proj"], None, self.x, self.q["x"].struct, stream)
        hh.hh_mx_product(ctx, self.fwd_cfg, self.q["x"].struct, self.q["w"].struct, self.branch, False, ws, stream)
        hh.hh_add_norm_fwd(ctx, self.norm_cfg, self._drop(use), y, self.branch, self.w["g_norm"], self.sum, self.normed, None, stream)
        return self.normed

    def backward(self, ctx, y, dn, dy, use: int, accumulate: bool, ws, stream) -> None:
        """dy (may be dn) from dn, the gradient of forward's result; the parameters' gradients are written, or added to."""
        if not self.projects:
            hh.hh_add_norm_bwd(ctx, self.norm_cfg, None, y, self.w["g_norm"], dn, None, dy, None, self.g["g_norm"], accumulate, ws, stream)
            return
        h, f = self.hidden, self.format
        hh.hh_add_norm_bwd(ctx, self.norm_cfg, self._drop(use), self.sum, self.w["g_norm"], dn, None, dy, self.dbranch, self.g["g_norm"], accumulate, ws,
                           stream)
        hh.hh_mx_quantise(ctx, self.tokens, h, self.dtype, self.dbranch, h, f, self.q["d"].struct, self.q["d_t"].struct, stream)
        hh.hh_mx_quantise(ctx, self.tokens, h, self.dtype, self.x, h, f, None, self.q["x_t"].struct, stream)
        hh.hh_mx_product(ctx, self.fwd_cfg, self.q["d"].struct, self.q["w_t"].struct, self.dx, False, ws, stream)
        hh.hh_mx_product(ctx, self.weight_cfg, self.q["d_t"].struct, self.q["x_t"].struct, self.g["w_proj"], accumulate, ws, stream)
        hh.hh_add_norm_bwd(ctx, self.proj_cfg, None, y, self.w["g_proj"], self.dx, dy, dy, None, self.g["g_proj"], accumulate, ws, stream)
