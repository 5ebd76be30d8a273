"""A pre-norm attention layer over the voxels of packed scans, on the libspv C ABI.

    h = layer_norm(x),  q = h Wq,  k = h Wk,  v = h Wv,  y = x + attention(q, k, v) Wo

The sparse convolutions mix a voxel with its 26 neighbours; this layer lets every voxel of a scan read every
other, as one does at a network's coarse strides, where a scan has a few thousand.  Scores may fall with the
voxels' L1 distance (a slope for each head) and be capped by a tanh, and a key head may serve several query
heads.  A few tokens of their own (a scan's summary, say) may take the voxels' place as queries.

Every step runs in libspv's kernels; the module only sequences the calls and holds the buffers.
"""
from __future__ import annotations

import threading
from typing import Dict, Optional

import torch

from . import spv


def scan_offsets(coords: torch.Tensor, scans: int) -> torch.Tensor:
    """[scans + 1] int32: the first row of each scan in a voxel list [m][4] in canonical order (no
    synchronization); a scan without voxels has an empty range."""
    b = coords[:, 0].contiguous()
    return torch.searchsorted(b, torch.arange(scans + 1, dtype=b.dtype, device=b.device), out_int32=True)


def _rows(t: torch.Tensor, width: int, dtype: torch.dtype, name: str, rows: Optional[int] = None):
    """Refuses what the calls would read past: t must be contiguous [rows][width] of dtype."""
    if t.dim() != 2 or t.shape[1] != width or t.dtype != dtype or not t.is_contiguous() or \
            (rows is not None and t.shape[0] != rows):
        raise ValueError(f"{name} must be contiguous [{'rows' if rows is None else rows}][{width}] of {dtype}")


class ScanAttention:
    """params: gamma, beta [C] f32; Wq [C][H D], Wk, Wv [C][Hkv D], Wo [H D][C] of the features' type.

    Calls on several streams or from several threads may overlap: the layer keeps workspaces for each."""

    def __init__(self, params: Dict[str, torch.Tensor], heads: int, kv_heads: Optional[int] = None, cap: float = 0.0,
                 slopes: Optional[torch.Tensor] = None, eps: float = 1e-5):
        self.P = {n: t.contiguous() for n, t in params.items()}
        self.C, width = self.P["Wq"].shape
        self.H, self.K = heads, heads if kv_heads is None else kv_heads
        if self.H <= 0 or self.K <= 0 or self.H % self.K:
            raise ValueError("heads must be a multiple of the key heads")
        if width % heads or self.P["Wk"].shape != (self.C, self.K * (width // heads)) or \
                self.P["Wv"].shape != self.P["Wk"].shape or self.P["Wo"].shape != (width, self.C):
            raise ValueError("the weights do not fit the heads")
        self.D, self.dtype = width // heads, self.P["Wq"].dtype
        if self.dtype not in (torch.float32, torch.bfloat16, torch.float16) or \
                any(self.P[n].dtype != self.dtype for n in ("Wk", "Wv", "Wo")):
            raise ValueError("the weights must be of one type, float32, bfloat16 or float16")
        for n, t in (("gamma", self.P["gamma"]), ("beta", self.P["beta"]), ("slopes", slopes)):
            size = heads if n == "slopes" else self.C
            if t is not None and (t.dtype != torch.float32 or t.shape != (size,)):
                raise ValueError(f"{n} must be float32 [{size}]")
        self.cap, self.slopes, self.eps = cap, slopes, eps
        self.ws: Dict[tuple, tuple] = {}

    def _ws(self, name: str, sizes: tuple, make) -> spv.Workspace:
        """The current stream's and thread's workspace `name` for a call of these sizes: the last one where it served
        them, or is large enough."""
        key = (name, spv._stream().value, threading.get_ident())
        last = self.ws.get(key)
        if last is None or last[0] != sizes:
            w = make()
            last = self.ws[key] = (sizes, w if last is None or w.nbytes > last[1].nbytes else last[1])
        return last[1]

    def _linear(self, x, W, res=None):
        sizes = (max(x.shape[0], 1), max(self.C, self.H * self.D))
        ws = self._ws("ops", sizes, lambda: spv.Workspace.for_ops(*sizes))
        return spv.spv_linear(ws, x, W, res=res)[: x.shape[0]]

    def _attention_ws(self, p, m, n, dtype):
        return self._ws("attention", (m, n, p.B), lambda: spv.Workspace.for_attention_backward(p, m, n, dtype))

    def forward(self, x: torch.Tensor, off: torch.Tensor, coords: Optional[torch.Tensor] = None,
                tokens: Optional[torch.Tensor] = None, token_off: Optional[torch.Tensor] = None,
                token_coords: Optional[torch.Tensor] = None, save: Optional[dict] = None) -> torch.Tensor:
        """y [m][C]: of the voxels x [n][C] themselves, or of tokens [m][C] whose scans' ranges are token_off.
        save (a dict): receives what backward() reads."""
        P, own = self.P, tokens is None
        t = x if own else tokens
        _rows(x, self.C, self.dtype, "x")
        if not own:
            _rows(tokens, self.C, self.dtype, "tokens")
            if token_off is None:
                raise ValueError("tokens come with their scans' ranges, token_off")
        n, m = x.shape[0], t.shape[0]
        if self.slopes is not None:
            for c, r, name in ((coords, n, "coords"),) if own else ((coords, n, "coords"), (token_coords, m, "token_coords")):
                if c is None or c.dtype != torch.int32 or c.dim() != 2 or c.shape[1] != 4 or c.shape[0] < r:
                    raise ValueError(f"slopes come with {name}, int32 [{r}][4]")
        h = spv.spv_layer_norm(x, P["gamma"], P["beta"], self.eps)
        ht = h if own else spv.spv_layer_norm(t, P["gamma"], P["beta"], self.eps)
        q = self._linear(ht, P["Wq"]).view(m, self.H, self.D)
        k = self._linear(h, P["Wk"]).view(n, self.K, self.D)
        v = self._linear(h, P["Wv"]).view(n, self.K, self.D)
        bias = self.slopes is not None
        p = spv.make_attention_params(self.H, self.K, self.D, off if own else token_off, off, cap=self.cap,
                                      q_coords=(coords if own else token_coords) if bias else None,
                                      k_coords=coords if bias else None, slopes=self.slopes)
        ws = self._attention_ws(p, m, n, x.dtype)
        if save is None:
            o = spv.spv_attention(ws, p, q, k, v)
        else:
            o, lse = spv.spv_attention(ws, p, q, k, v, want_lse=True)
            save.update(x=x, h=h, q=q, k=k, v=v, o=o, lse=lse, p=p, own=own)
        return self._linear(o.view(m, self.H * self.D), P["Wo"], res=t)

    def backward(self, saved: dict, dy: torch.Tensor) -> Dict[str, torch.Tensor]:
        """Gradients of x and of every parameter (weights, gamma and beta in float32), for the voxels' own queries."""
        if not saved["own"]:
            raise ValueError("backward takes the voxels' own queries")
        P, x, h, p = self.P, saved["x"], saved["h"], saved["p"]
        n, width, kv = x.shape[0], self.H * self.D, self.K * self.D
        _rows(dy, self.C, self.dtype, "dy", n)
        g = {}
        wide = (max(self.C, width), max(self.C, width))
        lin = self._ws("linear", wide, lambda: spv.Workspace.for_linear_backward(*wide))
        do, g["Wo"] = spv.spv_linear_backward(lin, saved["o"].view(n, width), P["Wo"], dy)
        ws = self._attention_ws(p, n, n, x.dtype)
        dq, dk, dv = spv.spv_attention_backward(ws, p, saved["q"], saved["k"], saved["v"], saved["o"], saved["lse"],
                                                do[:n].view(n, self.H, self.D))
        dh = None
        for name, d, w in (("Wq", dq, width), ("Wk", dk, kv), ("Wv", dv, kv)):
            d = d.view(n, w)
            _, g[name] = spv.spv_linear_backward(lin, h, P[name], d, want_dx=False)
            # The three products add up in the residual.  In 16 bits each sum is rounded (bf16 off by 2.3e-3, one rounding
            # 1.7e-3): the linear kernel takes up to 256 inputs, so not the three side by side.
            dh = self._linear(d, P[name].t().contiguous(), res=dh)
        wn = self._ws("norm", (n,), lambda: spv.Workspace.for_layer_norm_backward(n, self.C))
        g["x"], g["gamma"], g["beta"] = spv.spv_layer_norm_backward(wn, dh, x, P["gamma"], self.eps, dres=dy)
        return g
