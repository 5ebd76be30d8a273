"""A pre-activation residual layer on the voxels of packed scans, on the libspv C ABI.

    a = act(group_norm(x)),  u = a W1,  b = act(group_norm(u)),  y = x + b W2

The statistics are of a scan's voxels and a group's channels, so a scan's output does not depend on what else is in its
batch, and a batch may be one scan.  What the backward reads of x, a, u and b may be kept in 8 bits.

Every step runs in libspv's kernels; the module only sequences the calls and holds the buffers.
"""
from __future__ import annotations

from typing import Dict, Optional

import torch

from . import spv
from .scan_attention import ScanLayer, _rows


class ScanMLP(ScanLayer):
    """params: gamma1, beta1 [C] and gamma2, beta2 [F] f32; W1 [C][F], W2 [F][C] of the features' type.  act is "none",
    "relu" or "silu"; keep8: save holds rows in 8 bits (half of bf16's).  Contiguous parameters are read where they are, others
    copied once.

    16-bit products run on the matrix cores from a multiple of 8 channels, up to 128 or 225 to 256, to 16, 32, 64, 96, 128 or 256;
    others and float32's on a vector kernel."""

    def __init__(self, params: Dict[str, torch.Tensor], groups: int, act: str = "silu", eps: float = 1e-5,
                 keep8: bool = False):
        super().__init__()
        self.P = {n: t.contiguous() for n, t in params.items()}
        self.C, self.F = self.P["W1"].shape
        self.dtype = self.P["W1"].dtype
        if self.P["W2"].shape != (self.F, self.C) or self.P["W2"].dtype != self.dtype or \
                self.dtype not in (torch.float32, torch.bfloat16, torch.float16):
            raise ValueError("W1 [C][F] and W2 [F][C] must be of one type, float32, bfloat16 or float16")
        for n, size in (("gamma1", self.C), ("beta1", self.C), ("gamma2", self.F), ("beta2", self.F)):
            if self.P[n].dtype != torch.float32 or self.P[n].shape != (size,):
                raise ValueError(f"{n} must be float32 [{size}]")
        if groups <= 0 or self.C % groups or self.F % groups:
            raise ValueError("both widths must be multiples of the groups")
        if act not in ("none", "relu", "silu"):
            raise ValueError("act must be none, relu or silu")
        self.groups, self.act, self.eps, self.keep8 = groups, act, eps, keep8

    def _norm_ws(self, m: int, scans: int):
        wide = (m, max(self.C, self.F), self.groups, scans)

        def make():  # for both widths
            return max((spv.Workspace.for_group_norm_backward(m, w, self.groups, scans) for w in {self.C, self.F}),
                       key=lambda w: w.nbytes)
        return self._ws("group norm", wide, make)

    def _norm(self, x, off, layer: str, save: Optional[dict]):
        P, m = self.P, x.shape[0]
        got = spv.spv_group_norm(self._norm_ws(m, off.shape[0] - 1), x, off, self.groups, P["gamma" + layer],
                                 P["beta" + layer], self.eps, self.act, want_stat=save is not None,
                                 want_checkpoint=save is not None and self.keep8)
        if save is None:
            return got
        save["stat" + layer], save["in" + layer] = got[1], got[2] if self.keep8 else x
        save["out" + layer] = spv.spv_checkpoint8(got[0]) if self.keep8 else got[0]
        return got[0]

    def forward(self, x: torch.Tensor, off: torch.Tensor, save: Optional[dict] = None) -> torch.Tensor:
        """y [n][C] of the voxels x [n][C], whose scans' ranges are off [scans + 1] and hold every row.  save (a dict):
        receives what backward() reads."""
        _rows(x, self.C, self.dtype, "x")
        u = self._product(self._norm(x, off, "1", save), self.P["W1"], widest=max(self.C, self.F))
        b = self._norm(u, off, "2", save)
        if save is not None:
            save["off"] = off
        return self._product(b, self.P["W2"], res=x, widest=max(self.C, self.F))

    def backward(self, saved: dict, dy: torch.Tensor) -> Dict[str, torch.Tensor]:
        """Gradients of x and of every parameter (weights, gammas and betas in float32)."""
        P, off, g = self.P, saved["off"], {}
        kept = saved["in1"]
        m = (kept.codes if isinstance(kept, spv.Checkpoint8) else kept).shape[0]
        _rows(dy, self.C, self.dtype, "dy", m)
        ws, d, wide = self._norm_ws(m, off.shape[0] - 1), dy, max(self.C, self.F)
        for n in ("2", "1"):
            W = P["W" + n]
            g["W" + n] = self._weight_gradient(saved["out" + n], W, d, wide)
            d = self._product(d, W.t().contiguous(), widest=wide)
            d, g["gamma" + n], g["beta" + n] = spv.spv_group_norm_backward(
                ws, d, saved["in" + n], off, self.groups, saved["stat" + n], P["gamma" + n], P["beta" + n], self.act,
                dres=dy if n == "1" else None)
        g["x"] = d
        return g
