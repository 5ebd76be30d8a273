"""Python binding of libspv.so (ctypes): argument marshalling only.

Every function below forwards to the C entry point of the same name in
``include/spv.h``; all computation happens in the library's HIP kernels.
torch supplies device memory (tensor ``data_ptr``) and the stream
(``torch.cuda.current_stream().cuda_stream``).  Output tensors are allocated
here with torch when the caller does not pass them.

There is no fallback: if ``libspv.so`` is missing, or the tensors are not on a
GPU, the call raises.
"""
from __future__ import annotations

import ctypes as ct
import os
from dataclasses import dataclass
from typing import Optional, Sequence

import torch

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "libspv.so")

SPV_OK, SPV_ERR_INVALID_ARG, SPV_ERR_CAPACITY, SPV_ERR_RANGE, SPV_ERR_NONFINITE, SPV_ERR_UNSUPPORTED, SPV_ERR_HIP = \
    range(7)
SPV_F32, SPV_BF16, SPV_F16 = 0, 1, 2
SPV_DEVOX_CENTER, SPV_DEVOX_CORNER, SPV_DEVOX_NEAREST = 0, 1, 2
SPV_CHECKPOINT8_BLOCK = 32

_ACT = {"none": 0, "relu": 1, "silu": 2}
_DT = {torch.float32: SPV_F32, torch.bfloat16: SPV_BF16, torch.float16: SPV_F16}

# every symbol include/spv.h declares
EXPORTS = ("spv_workspace_bytes", "spv_voxelize", "spv_voxelize_onto", "spv_packed_weights_bytes",
           "spv_pack_weights", "spv_devoxelize_nbr", "spv_sparse_conv_nbr_packed", "spv_sparse_conv_up_packed", "spv_linear_packed",
           "spv_kernel_map", "spv_sparse_conv", "spv_sparse_conv_sliced",
           "spv_linear", "spv_kernel_map_nbr", "spv_sparse_conv_nbr", "spv_map_children", "spv_sparse_conv_up",
           "spv_sparse_conv_dgrad", "spv_sparse_conv_dgrad_nbr", "spv_wgrad_workspace_bytes", "spv_sparse_conv_wgrad",
           "spv_voxelize_backward",
           "spv_devoxelize_backward_workspace_bytes", "spv_devoxelize_backward", "spv_devoxelize",
           "spv_epilogue_backward_workspace_bytes", "spv_epilogue_backward",
           "spv_linear_backward_workspace_bytes", "spv_linear_backward",
           "spv_layer_norm", "spv_layer_norm_backward_workspace_bytes", "spv_layer_norm_backward",
           "spv_attention_workspace_bytes", "spv_attention", "spv_attention_backward_workspace_bytes",
           "spv_attention_backward", "spv_rope",
           "spv_checkpoint8", "spv_checkpoint8_read", "spv_linear_backward8_workspace_bytes", "spv_linear_backward8",
           "spv_group_norm_workspace_bytes", "spv_group_norm", "spv_group_norm_backward_workspace_bytes",
           "spv_group_norm_backward",
           "spv_block_workspace_bytes", "spv_block", "spv_lookup", "spv_voxel_lookup", "spv_conv_kernel",
           "spv_sparse_conv_nbr_noalloc",
           "spv_block_conv_kernel", "spv_status_check", "spv_status_string", "spv_last_hip_error")


class SpvError(RuntimeError):
    def __init__(self, status: int, what: str):
        self.status = status
        msg = lib().spv_status_string(status).decode() if _lib is not None else str(status)
        super().__init__(f"{what}: {msg} (status {status})")


class BlockParams(ct.Structure):
    _fields_ = [("C", ct.c_int32), ("dtype", ct.c_int32), ("voxel_size", ct.c_float), ("n_convs", ct.c_int32),
                ("W", ct.c_void_p * 2), ("scale", ct.c_void_p * 2), ("shift", ct.c_void_p * 2),
                ("relu", ct.c_int32 * 2), ("Wp", ct.c_void_p), ("scale_p", ct.c_void_p), ("shift_p", ct.c_void_p),
                ("relu_p", ct.c_int32), ("devox_mode", ct.c_int32), ("residual", ct.c_int32),
                ("events", ct.POINTER(ct.c_void_p)),
                ("n_events", ct.c_int32)]


class AttentionParams(ct.Structure):
    _fields_ = [("H", ct.c_int32), ("Hkv", ct.c_int32), ("D", ct.c_int32), ("B", ct.c_int32), ("scale", ct.c_float),
                ("cap", ct.c_float), ("q_off", ct.c_void_p), ("k_off", ct.c_void_p), ("q_coords", ct.c_void_p),
                ("k_coords", ct.c_void_p), ("slopes", ct.c_void_p)]


class RopeParams(ct.Structure):
    _fields_ = [("D", ct.c_int32), ("sections", ct.c_int32 * 3), ("halves", ct.c_int32), ("freqs", ct.c_void_p)]


_lib = None


def lib():
    """Load libspv.so (raises if it has not been built)."""
    global _lib
    if _lib is None:
        if not os.path.exists(LIB_PATH):
            raise RuntimeError(f"{LIB_PATH} is missing: build it with `python -m paper_2007_16100_amd.build`")
        L = ct.CDLL(LIB_PATH)
        vp, i64, i32, f32, sz = ct.c_void_p, ct.c_int64, ct.c_int32, ct.c_float, ct.c_size_t
        L.spv_workspace_bytes.argtypes = [i64, i32]
        L.spv_workspace_bytes.restype = sz
        L.spv_block_workspace_bytes.argtypes = [i64, i32]
        L.spv_block_workspace_bytes.restype = sz
        L.spv_voxelize.argtypes = [vp, vp, sz, vp, vp, i64, f32, vp, i32, i32, vp, vp, vp, vp, vp, vp]
        L.spv_packed_weights_bytes.argtypes = [i32, i32, i32]
        L.spv_packed_weights_bytes.restype = sz
        L.spv_pack_weights.argtypes = [vp, vp, i32, i32, i32, i32, i32, i32, vp, sz]
        L.spv_sparse_conv_nbr_packed.argtypes = [vp, vp, sz, vp, i64, i32, vp, vp, vp, vp, vp, i32, vp, vp, i64, i32,
                                                 i32]
        L.spv_sparse_conv_up_packed.argtypes = [vp, vp, sz, vp, vp, i64, i32, vp, vp, vp, vp, vp, i32, vp, i64, i32,
                                                i32]
        L.spv_linear_packed.argtypes = [vp, vp, sz, vp, vp, i64, i32, vp, vp, vp, i32, vp, i32, vp, i32, i32]
        L.spv_voxelize_onto.argtypes = [vp, vp, sz, vp, vp, i64, vp, vp, i64, f32, vp, i32, i32, vp, vp, vp]
        L.spv_kernel_map.argtypes = [vp, vp, sz, vp, vp, i64, i32, i32, vp, vp, vp, vp, i64, vp]
        L.spv_sparse_conv.argtypes = [vp, vp, sz, vp, i64, i32, vp, vp, i64, i32, i32, vp, vp, vp, i32, vp, vp, i64,
                                      i32, i32]
        L.spv_sparse_conv_sliced.argtypes = [vp, vp, sz, vp, i64, i32, vp, vp, i64, i32, i32, vp, i32, i32, vp, vp,
                                             vp, i32, vp, vp, i64, i32, i32]
        L.spv_linear.argtypes = [vp, vp, sz, vp, vp, i64, i32, vp, i32, i32, vp, vp, i32, vp, i32, vp, i32, i32]
        L.spv_kernel_map_nbr.argtypes = [vp, vp, sz, vp, vp, i64, vp]
        L.spv_sparse_conv_nbr.argtypes = [vp, vp, sz, vp, i64, i32, vp, vp, i32, i32, vp, vp, vp, i32, vp, vp, i64, i32,
                                          i32]
        L.spv_map_children.argtypes = [vp, vp, sz, vp, vp, i64, i64, vp, i64, vp]
        L.spv_sparse_conv_up.argtypes = [vp, vp, sz, vp, vp, i64, i32, vp, vp, i32, i32, vp, vp, vp, i32, vp, i64, i32,
                                         i32]
        L.spv_sparse_conv_dgrad.argtypes = [vp, vp, sz, vp, i64, i32, vp, vp, i64, i32, i32, vp, vp, vp, i64, i32, i32]
        L.spv_sparse_conv_dgrad_nbr.argtypes = [vp, vp, sz, vp, i32, vp, vp, vp, vp, i64, i32, i32]
        L.spv_sparse_conv_wgrad.argtypes = [vp, vp, sz, vp, i64, i32, vp, i64, i32, vp, vp, i64, i32, i32, vp, i32]
        L.spv_wgrad_workspace_bytes.argtypes = [i32, i32, i32]
        L.spv_wgrad_workspace_bytes.restype = sz
        L.spv_voxelize_backward.argtypes = [vp, vp, i64, i32, vp, vp, i64, vp, i32]
        L.spv_devoxelize_backward.argtypes = [vp, vp, sz, vp, vp, vp, i64, i32, vp, i64, i32]
        L.spv_devoxelize_backward_workspace_bytes.argtypes = [i64, i64]
        L.spv_epilogue_backward_workspace_bytes.argtypes = [i64, i32]
        L.spv_epilogue_backward_workspace_bytes.restype = sz
        L.spv_epilogue_backward.argtypes = [vp, vp, sz, vp, vp, vp, vp, i32, vp, i32, i64, i32, vp, vp, vp, vp, i32]
        L.spv_linear_backward_workspace_bytes.argtypes = [i32, i32]
        L.spv_linear_backward_workspace_bytes.restype = sz
        L.spv_linear_backward.argtypes = [vp, vp, sz, vp, i64, i32, vp, i32, vp, vp, vp, i32]
        L.spv_devoxelize_backward_workspace_bytes.restype = sz
        L.spv_layer_norm.argtypes = [vp, vp, vp, i64, i32, vp, vp, f32, vp, i32]
        L.spv_layer_norm_backward_workspace_bytes.argtypes = [i64, i32]
        L.spv_layer_norm_backward_workspace_bytes.restype = sz
        L.spv_layer_norm_backward.argtypes = [vp, vp, sz, vp, vp, vp, i64, i32, vp, f32, vp, vp, vp, vp, i32]
        ap = ct.POINTER(AttentionParams)
        for f in ("spv_attention_workspace_bytes", "spv_attention_backward_workspace_bytes"):
            getattr(L, f).argtypes = [ap, i64, i64, i32]
            getattr(L, f).restype = sz
        L.spv_attention.argtypes = [vp, vp, sz, ap, vp, i64, i64, vp, i64, vp, i64, i64, vp, i64, vp, i32]
        L.spv_attention_backward.argtypes = [vp, vp, sz, ap, vp, i64, i64, vp, i64, vp, i64, i64, vp, i64, vp, vp, i64,
                                             vp, i64, vp, i64, vp, i64, i32]
        L.spv_rope.argtypes = [vp, ct.POINTER(RopeParams), vp, vp, i64, vp, i64, i32, vp, i64, i32, vp, i64, vp, i64, i32,
                               i32]
        L.spv_checkpoint8.argtypes = [vp, vp, vp, i64, i32, vp, vp, i32]
        L.spv_checkpoint8_read.argtypes = [vp, vp, vp, vp, i64, i32, vp, i32]
        L.spv_linear_backward8_workspace_bytes.argtypes = [i64, i32, i32]
        L.spv_linear_backward8_workspace_bytes.restype = sz
        L.spv_linear_backward8.argtypes = [vp, vp, sz, vp, vp, vp, i64, i32, vp, i32, vp, i32]
        for f in ("spv_group_norm_workspace_bytes", "spv_group_norm_backward_workspace_bytes"):
            getattr(L, f).argtypes = [i64, i32, i32, i32]
            getattr(L, f).restype = sz
        L.spv_group_norm.argtypes = [vp, vp, sz, vp, i64, i32, vp, i32, i32, vp, vp, f32, i32, vp, vp, vp, vp, i32]
        L.spv_group_norm_backward.argtypes = [vp, vp, sz, vp, vp, vp, vp, i64, i32, vp, i32, i32, vp, vp, vp, i32, vp,
                                              vp, vp, vp, i32]
        L.spv_devoxelize.argtypes = [vp, vp, sz, vp, vp, i64, i32, vp, vp, i64, f32, i32, vp, i32, vp, i32, vp, vp,
                                     vp, i32, vp, i32, vp, vp]
        L.spv_devoxelize_nbr.argtypes = [vp, vp, sz, vp, vp, i64, vp, vp, i32, vp, vp, i64, f32, i32, vp, i32, vp,
                                         i32, vp, vp, vp, i32, vp, i32]
        L.spv_block.argtypes = [vp, vp, sz, ct.POINTER(BlockParams), vp, vp, i64, vp, vp, vp]
        L.spv_lookup.argtypes = [vp, vp, sz, vp, vp, i64, vp, i64, vp]
        L.spv_voxel_lookup.argtypes = [vp, vp, sz, i64, vp, i64, vp]
        L.spv_sparse_conv_nbr_noalloc.argtypes = [vp, vp, i64, i32, vp, vp, i32, i32, vp, vp, vp, i32, vp, vp, i64,
                                                  i32, i32]
        L.spv_conv_kernel.argtypes = [i32, i32, i32, i32, i64, i64, i64, i32]
        L.spv_conv_kernel.restype = i32
        L.spv_block_conv_kernel.argtypes = [i64, i32, i32]
        L.spv_block_conv_kernel.restype = i32
        L.spv_status_check.argtypes = [vp, vp]
        L.spv_status_string.argtypes = [i32]
        L.spv_status_string.restype = ct.c_char_p
        L.spv_last_hip_error.argtypes = []
        for f in ("spv_voxelize", "spv_voxelize_onto", "spv_pack_weights", "spv_devoxelize_nbr", "spv_sparse_conv_nbr_packed",
                  "spv_sparse_conv_up_packed", "spv_linear_packed", "spv_kernel_map", "spv_sparse_conv", "spv_sparse_conv_sliced", "spv_linear",
                  "spv_kernel_map_nbr", "spv_sparse_conv_nbr", "spv_map_children", "spv_sparse_conv_up",
                  "spv_sparse_conv_dgrad", "spv_sparse_conv_dgrad_nbr", "spv_sparse_conv_wgrad",
                  "spv_voxelize_backward",
                  "spv_devoxelize_backward", "spv_epilogue_backward", "spv_linear_backward", "spv_devoxelize",
                  "spv_layer_norm", "spv_layer_norm_backward", "spv_attention", "spv_attention_backward", "spv_rope",
                  "spv_checkpoint8", "spv_checkpoint8_read", "spv_linear_backward8", "spv_group_norm",
                  "spv_group_norm_backward", "spv_block", "spv_lookup", "spv_voxel_lookup",
                  "spv_sparse_conv_nbr_noalloc", "spv_status_check"):
            getattr(L, f).restype = ct.c_int
        _lib = L
    return _lib


def _ptr(t: Optional[torch.Tensor]):
    if t is None:
        return None
    if not t.is_cuda:
        raise ValueError("libspv takes device tensors")
    if not t.is_contiguous():
        raise ValueError("libspv takes contiguous tensors")
    return ct.c_void_p(t.data_ptr())


# the current stream's handle without the Stream object that torch.cuda.current_stream builds (2.8 us a call)
_raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None)


def _stream():
    if _raw_stream is not None:
        return ct.c_void_p(_raw_stream(torch.cuda.current_device()))
    return ct.c_void_p(torch.cuda.current_stream().cuda_stream)


def _addr(t: Optional[torch.Tensor]):
    """_ptr as a plain integer, which the calls take as well."""
    if t is None:
        return None
    if not t.is_cuda:
        raise ValueError("libspv takes device tensors")
    if not t.is_contiguous():
        raise ValueError("libspv takes contiguous tensors")
    return t.data_ptr()


def _chk(st: int, what: str):
    if st != SPV_OK:
        raise SpvError(st, what)


class Workspace:
    """A caller-owned device workspace (a torch uint8 buffer, 256-byte aligned)."""

    def __init__(self, nbytes: int, device="cuda"):
        self.nbytes = int(nbytes)
        self.buf = torch.empty(self.nbytes + 256, dtype=torch.uint8, device=device)
        off = (-self.buf.data_ptr()) % 256
        self.ptr = ct.c_void_p(self.buf.data_ptr() + off)

    @classmethod
    def for_ops(cls, max_points: int, max_C: int, device="cuda"):
        return cls(lib().spv_workspace_bytes(max_points, max_C), device)

    @classmethod
    def for_wgrad(cls, K3: int, Cin: int, Cout: int, device="cuda"):
        return cls(lib().spv_wgrad_workspace_bytes(K3, Cin, Cout), device)

    @classmethod
    def for_devox_backward(cls, n: int, m: int, device="cuda"):
        return cls(lib().spv_devoxelize_backward_workspace_bytes(n, m), device)

    @classmethod
    def for_epilogue_backward(cls, m: int, C: int, device="cuda"):
        return cls(max(lib().spv_epilogue_backward_workspace_bytes(m, C), 256), device)

    @classmethod
    def for_linear_backward(cls, Cin: int, Cout: int, device="cuda"):
        return cls(lib().spv_linear_backward_workspace_bytes(Cin, Cout), device)

    @classmethod
    def for_layer_norm_backward(cls, m: int, C: int, device="cuda"):
        return cls(lib().spv_layer_norm_backward_workspace_bytes(m, C), device)

    @classmethod
    def for_attention(cls, params: "AttentionParams", nq: int, nk: int, dtype: torch.dtype, device="cuda"):
        return cls(lib().spv_attention_workspace_bytes(ct.byref(params), nq, nk, _DT[dtype]), device)

    @classmethod
    def for_attention_backward(cls, params: "AttentionParams", nq: int, nk: int, dtype: torch.dtype, device="cuda"):
        """Serves the forward call of the same sizes too."""
        need = max(lib().spv_attention_workspace_bytes(ct.byref(params), nq, nk, _DT[dtype]),
                   lib().spv_attention_backward_workspace_bytes(ct.byref(params), nq, nk, _DT[dtype]))
        return cls(need, device)

    @classmethod
    def for_linear_backward8(cls, m: int, Cin: int, Cout: int, device="cuda"):
        return cls(lib().spv_linear_backward8_workspace_bytes(m, Cin, Cout), device)

    @classmethod
    def for_group_norm(cls, m: int, C: int, groups: int, scans: int, device="cuda"):
        return cls(lib().spv_group_norm_workspace_bytes(m, C, groups, scans), device)

    @classmethod
    def for_group_norm_backward(cls, m: int, C: int, groups: int, scans: int, device="cuda"):
        """Serves the forward call of the same sizes too."""
        return cls(max(lib().spv_group_norm_workspace_bytes(m, C, groups, scans),
                       lib().spv_group_norm_backward_workspace_bytes(m, C, groups, scans)), device)

    @classmethod
    def for_block(cls, max_points: int, C: int, device="cuda"):
        return cls(lib().spv_block_workspace_bytes(max_points, C), device)


def spv_workspace_bytes(max_points: int, max_C: int) -> int:
    return lib().spv_workspace_bytes(max_points, max_C)


def spv_block_workspace_bytes(max_points: int, C: int) -> int:
    return lib().spv_block_workspace_bytes(max_points, C)


def spv_status_check(ws: Workspace) -> int:
    return lib().spv_status_check(ws.ptr, _stream())


@dataclass
class Voxelized:
    coords: torch.Tensor    # [cap, 4] int32
    vfeat: Optional[torch.Tensor]
    counts: torch.Tensor    # [cap] int32
    pt2vox: torch.Tensor    # [n] int32
    m_dev: torch.Tensor     # [1] int64 on device
    m: Optional[int]        # host copy when synchronized


def spv_voxelize(ws: Workspace, xyz: torch.Tensor, voxel_size: float, feat: Optional[torch.Tensor] = None,
                 batch: Optional[torch.Tensor] = None, sync: bool = True, out: Optional[Voxelized] = None
                 ) -> Voxelized:
    n = xyz.shape[0]
    dev = xyz.device
    C = feat.shape[1] if feat is not None else 0
    dt = _DT[feat.dtype] if feat is not None else SPV_F32
    cap = max(n, 1)
    if out is None:
        out = Voxelized(torch.empty((cap, 4), dtype=torch.int32, device=dev),
                        torch.empty((cap, C), dtype=feat.dtype, device=dev) if feat is not None else None,
                        torch.empty(cap, dtype=torch.int32, device=dev),
                        torch.empty(cap, dtype=torch.int32, device=dev),
                        torch.zeros(1, dtype=torch.int64, device=dev), None)
    m_host = ct.c_int64(0)
    st = lib().spv_voxelize(_stream(), ws.ptr, ws.nbytes, _ptr(xyz), _ptr(batch), n, ct.c_float(voxel_size),
                            _ptr(feat), C, dt, _ptr(out.coords), _ptr(out.vfeat), _ptr(out.counts), _ptr(out.pt2vox),
                            _ptr(out.m_dev), ct.byref(m_host) if sync else None)
    _chk(st, "spv_voxelize")
    out.m = m_host.value if sync else None
    return out


def spv_voxelize_onto(ws: Workspace, coords: torch.Tensor, xyz: torch.Tensor, voxel_size: float,
                      feat: Optional[torch.Tensor] = None, batch: Optional[torch.Tensor] = None,
                      m_dev: Optional[torch.Tensor] = None, out: Optional[Voxelized] = None) -> Voxelized:
    """Scatter-mean of the points onto the given voxel set (row j of the outputs is coords row j);
    points whose voxel is not in the set get pt2vox -1.  Returns a Voxelized whose coords are
    the given ones."""
    n = xyz.shape[0]
    m_cap = coords.shape[0]
    dev = xyz.device
    C = feat.shape[1] if feat is not None else 0
    dt = _DT[feat.dtype] if feat is not None else SPV_F32
    if out is None:
        out = Voxelized(coords, torch.empty((max(m_cap, 1), C), dtype=feat.dtype, device=dev)
                        if feat is not None else None,
                        torch.empty(max(m_cap, 1), dtype=torch.int32, device=dev),
                        torch.empty(max(n, 1), dtype=torch.int32, device=dev), m_dev,
                        m_cap if m_dev is None else None)
    st = lib().spv_voxelize_onto(_stream(), ws.ptr, ws.nbytes, _ptr(coords), _ptr(m_dev), m_cap, _ptr(xyz),
                                 _ptr(batch), n, ct.c_float(voxel_size), _ptr(feat), C, dt, _ptr(out.vfeat),
                                 _ptr(out.counts), _ptr(out.pt2vox))
    _chk(st, "spv_voxelize_onto")
    return out


@dataclass
class KernelMap:
    out_coords: Optional[torch.Tensor]
    m_out_dev: torch.Tensor
    off: torch.Tensor       # [K^3 + 1] int32
    pairs: torch.Tensor     # [pair_cap, 2] int32 (in, out)
    total: Optional[int]


def spv_kernel_map(ws: Workspace, in_coords: torch.Tensor, K: int = 3, stride: int = 1,
                   m_in_dev: Optional[torch.Tensor] = None, m_cap: Optional[int] = None,
                   pair_cap: Optional[int] = None, sync: bool = True) -> KernelMap:
    dev = in_coords.device
    m_cap = in_coords.shape[0] if m_cap is None else m_cap
    K3 = K ** 3
    if pair_cap is None:
        # K=2 s2: each input in one pair; K=3 s2: at most 2 outputs per odd axis
        pair_cap = max(1, m_cap if K == 2 else (8 * m_cap if stride == 2 else K3 * m_cap))
    oc = torch.empty((max(m_cap, 1), 4), dtype=torch.int32, device=dev) if stride == 2 else None
    km = KernelMap(oc, torch.zeros(1, dtype=torch.int64, device=dev), torch.empty(K3 + 1, dtype=torch.int32, device=dev),
                   torch.empty((pair_cap, 2), dtype=torch.int32, device=dev), None)
    tot = ct.c_int64(0)
    st = lib().spv_kernel_map(_stream(), ws.ptr, ws.nbytes, _ptr(in_coords), _ptr(m_in_dev), m_cap, K, stride,
                              _ptr(oc), _ptr(km.m_out_dev), _ptr(km.off), _ptr(km.pairs), pair_cap,
                              ct.byref(tot) if sync else None)
    if sync:
        km.total = tot.value
    _chk(st, "spv_kernel_map")
    return km


def spv_sparse_conv(ws: Workspace, x: torch.Tensor, off: torch.Tensor, pairs: torch.Tensor, W: torch.Tensor,
                    m_out_cap: int, m_out_dev: Optional[torch.Tensor] = None, scale: Optional[torch.Tensor] = None,
                    shift: Optional[torch.Tensor] = None, relu: bool = False, transposed: bool = False,
                    out: Optional[torch.Tensor] = None) -> torch.Tensor:
    K3, Cin, Cout = W.shape
    if out is None:
        out = torch.empty((max(m_out_cap, 1), Cout), dtype=x.dtype, device=x.device)
    st = lib().spv_sparse_conv(_stream(), ws.ptr, ws.nbytes, _ptr(x), x.shape[0], Cin, _ptr(off), _ptr(pairs),
                               pairs.shape[0], K3, int(transposed), _ptr(W), _ptr(scale), _ptr(shift), int(relu),
                               _ptr(out), _ptr(m_out_dev), m_out_cap, Cout, _DT[x.dtype])
    _chk(st, "spv_sparse_conv")
    return out


def spv_sparse_conv_sliced(ws: Workspace, x: torch.Tensor, off: torch.Tensor, pairs: torch.Tensor,
                           W_full: torch.Tensor, Cin: int, Cout: int, m_out_cap: int,
                           m_out_dev: Optional[torch.Tensor] = None, scale: Optional[torch.Tensor] = None,
                           shift: Optional[torch.Tensor] = None, relu: bool = False, transposed: bool = False,
                           out: Optional[torch.Tensor] = None, res: Optional[torch.Tensor] = None,
                           cin_offset: int = 0, in_rows: Optional[int] = None) -> torch.Tensor:
    """The conv with input channels cin_offset .. cin_offset+Cin and the first Cout output
    channels of the full weight W_full [K3][Cin_full][Cout_full] (and the first Cout entries of
    the full scale / shift); res: a residual input added before the activation."""
    K3, Cin_full, Cout_full = W_full.shape
    if x.shape[1] != Cin:
        raise ValueError(f"x has {x.shape[1]} channels, the slice takes {Cin}")
    if cin_offset < 0 or cin_offset + Cin > Cin_full:
        raise ValueError("input-channel slice outside the weight")
    if out is None:
        out = torch.empty((max(m_out_cap, 1), Cout), dtype=x.dtype, device=x.device)
    wp = ct.c_void_p(_ptr(W_full).value + cin_offset * Cout_full * W_full.element_size())
    st = lib().spv_sparse_conv_sliced(_stream(), ws.ptr, ws.nbytes, _ptr(x), x.shape[0] if in_rows is None else in_rows,
                                      Cin, _ptr(off), _ptr(pairs), pairs.shape[0], K3, int(transposed), wp,
                                      Cin_full, Cout_full, _ptr(scale),
                                      _ptr(shift), _ptr(res), int(relu), _ptr(out), _ptr(m_out_dev), m_out_cap, Cout,
                                      _DT[x.dtype])
    _chk(st, "spv_sparse_conv_sliced")
    return out


def spv_linear(ws: Workspace, x: torch.Tensor, W: torch.Tensor, Cout: Optional[int] = None,
               m_dev: Optional[torch.Tensor] = None, m_cap: Optional[int] = None,
               scale: Optional[torch.Tensor] = None, shift: Optional[torch.Tensor] = None, relu: bool = False,
               res: Optional[torch.Tensor] = None, res_after_act: bool = False, cin_offset: int = 0,
               out: Optional[torch.Tensor] = None) -> torch.Tensor:
    """act(scale * (x @ W[cin_offset : cin_offset + Cin, :Cout]) + shift [+ res]) [+ res]."""
    Cin = x.shape[1]
    Cin_full, Cout_full = W.shape
    Cout = Cout_full if Cout is None else Cout
    if cin_offset < 0 or cin_offset + Cin > Cin_full:
        raise ValueError("input-channel slice outside the weight")
    m_cap = x.shape[0] if m_cap is None else m_cap
    if out is None:
        out = torch.empty((max(m_cap, 1), Cout), dtype=x.dtype, device=x.device)
    wp = ct.c_void_p(_ptr(W).value + cin_offset * Cout_full * W.element_size())
    st = lib().spv_linear(_stream(), ws.ptr, ws.nbytes, _ptr(x), _ptr(m_dev), m_cap, Cin, wp, Cin_full - cin_offset,
                          Cout_full, _ptr(scale), _ptr(shift), int(relu), _ptr(res), int(res_after_act), _ptr(out),
                          Cout, _DT[x.dtype])
    _chk(st, "spv_linear")
    return out


def spv_pack_weights(W: torch.Tensor, Cin: Optional[int] = None, Cout: Optional[int] = None,
                     cin_offset: int = 0) -> Optional[torch.Tensor]:
    """The matrix-core fragments of W[:, cin_offset : cin_offset + Cin, :Cout] (W [K3][Cin_full][Cout_full],
    or [Cin_full][Cout_full] for a linear layer) as a uint8 device tensor, or None where no kernel
    reads that shape (and for float32)."""
    W3 = W if W.dim() == 3 else W.unsqueeze(0)
    K3, Cin_full, Cout_full = W3.shape
    Cin = Cin_full - cin_offset if Cin is None else Cin
    Cout = Cout_full if Cout is None else Cout
    if cin_offset < 0 or cin_offset + Cin > Cin_full:
        raise ValueError("input-channel slice outside the weight")
    nbytes = lib().spv_packed_weights_bytes(K3, Cin, Cout)
    if nbytes == 0 or W.dtype == torch.float32:
        return None
    out = torch.empty(nbytes, dtype=torch.uint8, device=W.device)
    wp = ct.c_void_p(_ptr(W3).value + cin_offset * Cout_full * W3.element_size())
    st = lib().spv_pack_weights(_stream(), wp, K3, Cin_full, Cout_full, Cin, Cout, _DT[W.dtype], _ptr(out), nbytes)
    _chk(st, "spv_pack_weights")
    return out


def spv_sparse_conv_nbr_packed(ws: Workspace, x: torch.Tensor, nbr: torch.Tensor, Wp: torch.Tensor, Cout: int,
                               m_out_cap: int, m_out_dev: Optional[torch.Tensor] = None,
                               scale: Optional[torch.Tensor] = None, shift: Optional[torch.Tensor] = None,
                               relu: bool = False, res: Optional[torch.Tensor] = None,
                               out: Optional[torch.Tensor] = None) -> torch.Tensor:
    """spv_sparse_conv_nbr with weights from spv_pack_weights (K3 = 27, x's width, Cout)."""
    if out is None:
        out = torch.empty((max(m_out_cap, 1), Cout), dtype=x.dtype, device=x.device)
    st = lib().spv_sparse_conv_nbr_packed(_stream(), ws.ptr, ws.nbytes, _ptr(x), x.shape[0], x.shape[1], _ptr(nbr),
                                          _ptr(Wp), _ptr(scale), _ptr(shift), _ptr(res), int(relu), _ptr(out),
                                          _ptr(m_out_dev), m_out_cap, Cout, _DT[x.dtype])
    _chk(st, "spv_sparse_conv_nbr_packed")
    return out


def spv_sparse_conv_up_packed(ws: Workspace, x: torch.Tensor, children: torch.Tensor, Wp: torch.Tensor, Cout: int,
                              out_rows: int, m_in_dev: Optional[torch.Tensor] = None,
                              scale: Optional[torch.Tensor] = None, shift: Optional[torch.Tensor] = None,
                              relu: bool = False, res: Optional[torch.Tensor] = None,
                              out: Optional[torch.Tensor] = None) -> torch.Tensor:
    """spv_sparse_conv_up with weights from spv_pack_weights (K3 = 8, x's width, Cout)."""
    if out is None:
        out = torch.empty((max(out_rows, 1), Cout), dtype=x.dtype, device=x.device)
    st = lib().spv_sparse_conv_up_packed(_stream(), ws.ptr, ws.nbytes, _ptr(x), _ptr(m_in_dev), x.shape[0],
                                         x.shape[1], _ptr(children), _ptr(Wp), _ptr(scale), _ptr(shift), _ptr(res),
                                         int(relu), _ptr(out), out_rows, Cout, _DT[x.dtype])
    _chk(st, "spv_sparse_conv_up_packed")
    return out


def spv_linear_packed(ws: Workspace, x: torch.Tensor, Wp: torch.Tensor, Cout: int,
                      m_dev: Optional[torch.Tensor] = None, m_cap: Optional[int] = None,
                      scale: Optional[torch.Tensor] = None, shift: Optional[torch.Tensor] = None, relu: bool = False,
                      res: Optional[torch.Tensor] = None, res_after_act: bool = False,
                      out: Optional[torch.Tensor] = None) -> torch.Tensor:
    """spv_linear with weights from spv_pack_weights (K3 = 1, x's width, Cout)."""
    m_cap = x.shape[0] if m_cap is None else m_cap
    if out is None:
        out = torch.empty((max(m_cap, 1), Cout), dtype=x.dtype, device=x.device)
    st = lib().spv_linear_packed(_stream(), ws.ptr, ws.nbytes, _ptr(x), _ptr(m_dev), m_cap, x.shape[1], _ptr(Wp),
                                 _ptr(scale), _ptr(shift), int(relu), _ptr(res), int(res_after_act), _ptr(out), Cout,
                                 _DT[x.dtype])
    _chk(st, "spv_linear_packed")
    return out


def spv_kernel_map_nbr(ws: Workspace, coords: torch.Tensor, m_dev: Optional[torch.Tensor] = None,
                       out: Optional[torch.Tensor] = None) -> torch.Tensor:
    """nbr [m][27] int32: entry k of row j is i + 1 for the voxel i at c_j + delta_k, else 0."""
    m_cap = coords.shape[0]
    if out is None:
        out = torch.empty((max(m_cap, 1), 27), dtype=torch.int32, device=coords.device)
    st = lib().spv_kernel_map_nbr(_stream(), ws.ptr, ws.nbytes, _ptr(coords), _ptr(m_dev), m_cap, _ptr(out))
    _chk(st, "spv_kernel_map_nbr")
    return out


def spv_sparse_conv_nbr(ws: Workspace, x: torch.Tensor, nbr: torch.Tensor, W_full: torch.Tensor, Cout: int,
                        m_out_cap: int, m_out_dev: Optional[torch.Tensor] = None, scale: Optional[torch.Tensor] = None,
                        shift: Optional[torch.Tensor] = None, relu: bool = False,
                        res: Optional[torch.Tensor] = None, cin_offset: int = 0,
                        out: Optional[torch.Tensor] = None) -> torch.Tensor:
    """The sliced conv (input channels cin_offset .. + x's width, first Cout outputs) on a
    neighbour table from spv_kernel_map_nbr."""
    K3, Cin_full, Cout_full = W_full.shape
    Cin = x.shape[1]
    if cin_offset < 0 or cin_offset + Cin > Cin_full:
        raise ValueError("input-channel slice outside the weight")
    if out is None:
        out = torch.empty((max(m_out_cap, 1), Cout), dtype=x.dtype, device=x.device)
    wp = ct.c_void_p(_ptr(W_full).value + cin_offset * Cout_full * W_full.element_size())
    st = lib().spv_sparse_conv_nbr(_stream(), ws.ptr, ws.nbytes, _ptr(x), x.shape[0], Cin, _ptr(nbr), wp, Cin_full,
                                   Cout_full, _ptr(scale), _ptr(shift), _ptr(res), int(relu), _ptr(out),
                                   _ptr(m_out_dev), m_out_cap, Cout, _DT[x.dtype])
    _chk(st, "spv_sparse_conv_nbr")
    return out


def spv_sparse_conv_nbr_noalloc(x: torch.Tensor, nbr: torch.Tensor, W_full: torch.Tensor, Cout: int,
                                m_out_cap: int, m_out_dev: Optional[torch.Tensor] = None,
                                scale: Optional[torch.Tensor] = None, shift: Optional[torch.Tensor] = None,
                                relu: bool = False, res: Optional[torch.Tensor] = None, cin_offset: int = 0,
                                out: Optional[torch.Tensor] = None) -> torch.Tensor:
    """spv_sparse_conv_nbr with no workspace (the library's device-resident scratch holds the
    packed weights); out must be given by callers that cannot allocate."""
    K3, Cin_full, Cout_full = W_full.shape
    Cin = x.shape[1]
    if cin_offset < 0 or cin_offset + Cin > Cin_full:
        raise ValueError("input-channel slice outside the weight")
    if out is None:
        out = torch.empty((max(m_out_cap, 1), Cout), dtype=x.dtype, device=x.device)
    wp = ct.c_void_p(_ptr(W_full).value + cin_offset * Cout_full * W_full.element_size())
    st = lib().spv_sparse_conv_nbr_noalloc(_stream(), _ptr(x), x.shape[0], Cin, _ptr(nbr), wp, Cin_full, Cout_full,
                                           _ptr(scale), _ptr(shift), _ptr(res), int(relu), _ptr(out),
                                           _ptr(m_out_dev), m_out_cap, Cout, _DT[x.dtype])
    _chk(st, "spv_sparse_conv_nbr_noalloc")
    return out


def spv_map_children(ws: Workspace, off: torch.Tensor, pairs: torch.Tensor, fine_rows: int, m_coarse: int,
                     m_coarse_dev: Optional[torch.Tensor] = None, out: Optional[torch.Tensor] = None) -> torch.Tensor:
    """children [m_coarse][8] int32 of a K=2 stride-2 map: fine row + 1 per offset, 0 = none."""
    if out is None:
        out = torch.empty((max(m_coarse, 1), 8), dtype=torch.int32, device=off.device)
    st = lib().spv_map_children(_stream(), ws.ptr, ws.nbytes, _ptr(off), _ptr(pairs), pairs.shape[0], fine_rows,
                                _ptr(m_coarse_dev), m_coarse, _ptr(out))
    _chk(st, "spv_map_children")
    return out


def spv_sparse_conv_up(ws: Workspace, x: torch.Tensor, children: torch.Tensor, W_full: torch.Tensor, Cout: int,
                       out_rows: int, m_in_dev: Optional[torch.Tensor] = None, scale: Optional[torch.Tensor] = None,
                       shift: Optional[torch.Tensor] = None, relu: bool = False, res: Optional[torch.Tensor] = None,
                       cin_offset: int = 0, out: Optional[torch.Tensor] = None) -> torch.Tensor:
    """The transposed k=2 s=2 conv of the coarse rows x onto the fine rows, from the child table."""
    K3, Cin_full, Cout_full = W_full.shape
    Cin = x.shape[1]
    if K3 != 8 or cin_offset < 0 or cin_offset + Cin > Cin_full:
        raise ValueError("W_full must be [8][Cin_full][Cout_full] holding the input-channel slice")
    if out is None:
        out = torch.empty((max(out_rows, 1), Cout), dtype=x.dtype, device=x.device)
    wp = ct.c_void_p(_ptr(W_full).value + cin_offset * Cout_full * W_full.element_size())
    st = lib().spv_sparse_conv_up(_stream(), ws.ptr, ws.nbytes, _ptr(x), _ptr(m_in_dev), x.shape[0], Cin,
                                  _ptr(children), wp, Cin_full, Cout_full, _ptr(scale), _ptr(shift), _ptr(res),
                                  int(relu), _ptr(out), out_rows, Cout, _DT[x.dtype])
    _chk(st, "spv_sparse_conv_up")
    return out


def spv_sparse_conv_dgrad(ws: Workspace, dy: torch.Tensor, off: torch.Tensor, pairs: torch.Tensor, W: torch.Tensor,
                          m_in_cap: int, m_in_dev: Optional[torch.Tensor] = None, transposed: bool = False,
                          out: Optional[torch.Tensor] = None) -> torch.Tensor:
    """dx[i] = sum over the pairs (i, j, k) of dy[j] @ W[k]^T (W: the forward weights [K3][Cin][Cout])."""
    K3, Cin, Cout = W.shape
    if out is None:
        out = torch.empty((max(m_in_cap, 1), Cin), dtype=dy.dtype, device=dy.device)
    st = lib().spv_sparse_conv_dgrad(_stream(), ws.ptr, ws.nbytes, _ptr(dy), dy.shape[0], Cout, _ptr(off), _ptr(pairs),
                                     pairs.shape[0], K3, int(transposed), _ptr(W), _ptr(out), _ptr(m_in_dev), m_in_cap,
                                     Cin, _DT[dy.dtype])
    _chk(st, "spv_sparse_conv_dgrad")
    return out


def spv_sparse_conv_wgrad(ws: Workspace, x: torch.Tensor, dy: torch.Tensor, off: torch.Tensor, pairs: torch.Tensor,
                          K3: int, transposed: bool = False, out: Optional[torch.Tensor] = None) -> torch.Tensor:
    """dW[k] = sum over the pairs (i, j) of offset k of x[i]^T dy[j], float32 [K3][Cin][Cout]."""
    Cin, Cout = x.shape[1], dy.shape[1]
    if out is None:
        out = torch.empty((K3, Cin, Cout), dtype=torch.float32, device=x.device)
    st = lib().spv_sparse_conv_wgrad(_stream(), ws.ptr, ws.nbytes, _ptr(x), x.shape[0], Cin, _ptr(dy), dy.shape[0],
                                     Cout, _ptr(off), _ptr(pairs), pairs.shape[0], K3, int(transposed), _ptr(out),
                                     _DT[x.dtype])
    _chk(st, "spv_sparse_conv_wgrad")
    return out


def spv_sparse_conv_dgrad_nbr(ws: Workspace, dy: torch.Tensor, nbr: torch.Tensor, W: torch.Tensor,
                              m_dev: Optional[torch.Tensor] = None, out: Optional[torch.Tensor] = None) -> torch.Tensor:
    """Input gradient of the 3x3x3 submanifold conv with weights W [27][Cin][Cout] on the neighbour table."""
    m_cap, Cout = dy.shape
    Cin = W.shape[1]
    if out is None:
        out = torch.empty((max(m_cap, 1), Cin), dtype=dy.dtype, device=dy.device)
    st = lib().spv_sparse_conv_dgrad_nbr(_stream(), ws.ptr, ws.nbytes, _ptr(dy), Cout, _ptr(nbr), _ptr(W), _ptr(out),
                                         _ptr(m_dev), m_cap, Cin, _DT[dy.dtype])
    _chk(st, "spv_sparse_conv_dgrad_nbr")
    return out


def spv_voxelize_backward(dvfeat: torch.Tensor, counts: torch.Tensor, pt2vox: torch.Tensor, m: int,
                          out: Optional[torch.Tensor] = None) -> torch.Tensor:
    n, C = pt2vox.shape[0], dvfeat.shape[1]
    if out is None:
        out = torch.empty((max(n, 1), C), dtype=dvfeat.dtype, device=dvfeat.device)
    st = lib().spv_voxelize_backward(_stream(), _ptr(dvfeat), m, C, _ptr(counts), _ptr(pt2vox), n, _ptr(out),
                                     _DT[dvfeat.dtype])
    _chk(st, "spv_voxelize_backward")
    return out


def spv_devoxelize_backward(ws: Workspace, corner_idx: torch.Tensor, corner_w: torch.Tensor, dout: torch.Tensor,
                            m: int, out: Optional[torch.Tensor] = None) -> torch.Tensor:
    n, C = dout.shape
    if out is None:
        out = torch.empty((max(m, 1), C), dtype=torch.float32, device=dout.device)
    st = lib().spv_devoxelize_backward(_stream(), ws.ptr, ws.nbytes, _ptr(corner_idx), _ptr(corner_w), _ptr(dout), n,
                                       C, _ptr(out), m, _DT[dout.dtype])
    _chk(st, "spv_devoxelize_backward")
    return out


def spv_epilogue_backward(ws: Workspace, dy: torch.Tensor, a: torch.Tensor, scale: Optional[torch.Tensor] = None,
                          shift: Optional[torch.Tensor] = None, relu: bool = False,
                          res: Optional[torch.Tensor] = None, res_after_act: bool = False):
    """(da, dres, dscale, dshift) of the epilogue act(scale * a + shift (+ res)) (+ res)."""
    m, C = dy.shape
    d = dy.device
    da = torch.empty((max(m, 1), C), dtype=dy.dtype, device=d)
    dres = torch.empty((max(m, 1), C), dtype=dy.dtype, device=d) if res is not None else None
    dscale = torch.empty(C, dtype=torch.float32, device=d)
    dshift = torch.empty(C, dtype=torch.float32, device=d)
    st = lib().spv_epilogue_backward(_stream(), ws.ptr, ws.nbytes, _ptr(dy), _ptr(a), _ptr(scale), _ptr(shift),
                                     int(relu), _ptr(res), int(res_after_act), m, C, _ptr(da), _ptr(dres),
                                     _ptr(dscale), _ptr(dshift), _DT[dy.dtype])
    _chk(st, "spv_epilogue_backward")
    return da, dres, dscale, dshift


def spv_linear_backward(ws: Workspace, x: torch.Tensor, W: torch.Tensor, da: torch.Tensor, want_dx: bool = True):
    """(dx, dW) of the product x @ W, given its gradient da; dx is None without want_dx."""
    m, Cin = x.shape
    Cout = W.shape[1]
    dx = torch.empty((max(m, 1), Cin), dtype=x.dtype, device=x.device) if want_dx else None
    dW = torch.empty((Cin, Cout), dtype=torch.float32, device=x.device)
    st = lib().spv_linear_backward(_stream(), ws.ptr, ws.nbytes, _ptr(x), m, Cin, _ptr(W), Cout, _ptr(da), _ptr(dx),
                                   _ptr(dW), _DT[x.dtype])
    _chk(st, "spv_linear_backward")
    return dx, dW


def spv_layer_norm(x: torch.Tensor, gamma: Optional[torch.Tensor] = None, beta: Optional[torch.Tensor] = None,
                   eps: float = 1e-5, m_dev: Optional[torch.Tensor] = None,
                   out: Optional[torch.Tensor] = None) -> torch.Tensor:
    """(x - mean) / sqrt(var + eps) * gamma + beta over the channels of each row of x [m][C]."""
    m, C = x.shape
    xp, gp, bp = _addr(x), _channels(gamma, C, "gamma"), _channels(beta, C, "beta")
    if out is None:
        out = torch.empty_like(x)
    elif out.shape != x.shape or out.dtype != x.dtype:
        raise ValueError("out must have x's shape and type")
    st = lib().spv_layer_norm(_stream(), xp, _addr(m_dev), m, C, gp, bp, eps, _addr(out), _DT[x.dtype])
    _chk(st, "spv_layer_norm")
    return out


def spv_layer_norm_backward(ws: Workspace, dy: torch.Tensor, x: torch.Tensor, gamma: Optional[torch.Tensor] = None,
                            eps: float = 1e-5, dres: Optional[torch.Tensor] = None,
                            m_dev: Optional[torch.Tensor] = None):
    """(dx, dgamma, dbeta) of spv_layer_norm; dres: a gradient added to dx (the residual branch's)."""
    m, C = x.shape
    xp, gp = _addr(x), _channels(gamma, C, "gamma")
    for t, name in ((dy, "dy"), (dres, "dres")):
        if t is not None and (t.shape != x.shape or t.dtype != x.dtype):
            raise ValueError(f"{name} must have x's shape and type")
    dx = torch.empty_like(x)
    dgamma = torch.empty(C, dtype=torch.float32, device=x.device)
    dbeta = torch.empty_like(dgamma)
    st = lib().spv_layer_norm_backward(_stream(), ws.ptr, ws.nbytes, _addr(dy), xp, _addr(m_dev), m, C, gp, eps,
                                       _addr(dres), dx.data_ptr(), dgamma.data_ptr(), dbeta.data_ptr(), _DT[x.dtype])
    _chk(st, "spv_layer_norm_backward")
    return dx, dgamma, dbeta


def _channels(t: Optional[torch.Tensor], C: int, name: str):
    """Address of a float32 vector of C entries (None: none)."""
    if t is None:
        return None
    if t.dtype != torch.float32 or t.shape != (C,):
        raise ValueError(f"{name} must be float32 [{C}]")
    return _addr(t)


def make_attention_params(H: int, Hkv: int, D: int, q_off: torch.Tensor, k_off: Optional[torch.Tensor] = None,
                          scale: Optional[float] = None, cap: float = 0.0, q_coords: Optional[torch.Tensor] = None,
                          k_coords: Optional[torch.Tensor] = None,
                          slopes: Optional[torch.Tensor] = None) -> AttentionParams:
    """Parameters of an attention over packed scans: scan b's queries are rows q_off[b] .. q_off[b+1] - 1 and
    its keys rows k_off[b] .. k_off[b+1] - 1 (int32 device tensors [B + 1]; k_off None: the queries' own).
    scale None: 1 / sqrt(D).  With slopes [H] and the rows' voxel coordinates [n][4] (k_coords None: the
    queries' own) a score falls by its head's slope times the L1 distance.

    The struct holds raw device pointers; it also keeps references to every tensor it points into, so
    they stay allocated as long as the struct lives."""
    if k_off is None:
        k_off = q_off
    if slopes is not None and k_coords is None:
        k_coords = q_coords
    for t, name in ((q_off, "q_off"), (k_off, "k_off")):
        if t.dtype != torch.int32 or t.dim() != 1 or t.shape != q_off.shape or t.shape[0] < 1:
            raise ValueError(f"{name} must be int32 [scans + 1]")
    for t, name in ((q_coords, "q_coords"), (k_coords, "k_coords")):
        if (t is None) != (slopes is None):
            raise ValueError("coordinates and slopes go together")
        if t is not None and (t.dtype != torch.int32 or t.dim() != 2 or t.shape[1] != 4):
            raise ValueError(f"{name} must be int32 [rows][4]")
    p = AttentionParams(H, Hkv, D, q_off.shape[0] - 1, D ** -0.5 if scale is None else scale, cap, _addr(q_off),
                        _addr(k_off), _addr(q_coords), _addr(k_coords), _channels(slopes, H, "slopes"))
    p._keep = (q_off, k_off, q_coords, k_coords, slopes)
    return p


def _heads(t: torch.Tensor, heads: int, D: int, dtype: torch.dtype, name: str):
    """(rows, address, row stride) of t [n][heads][D], whose rows may be parts of wider ones."""
    n, h, d = t.shape
    if h != heads or d != D or t.dtype != dtype:
        raise ValueError(f"{name} must be [rows][{heads}][{D}] of {dtype}")
    if not t.is_cuda:
        raise ValueError("libspv takes device tensors")
    ld, sh, sd = t.stride()
    if n and ((d > 1 and sd != 1) or (h > 1 and sh != d)):
        raise ValueError(f"the channels of a row of {name} must be contiguous")
    return n, t.data_ptr(), ld if n > 1 else h * d


def _qkv(p: AttentionParams, q, k, v):
    D, K, dt = p.D, p.Hkv, q.dtype
    nq, qp, ldq = _heads(q, p.H, D, dt, "q")
    nk, kp, ldk = _heads(k, K, D, dt, "k")
    nv, vp, ldv = _heads(v, K, D, dt, "v")
    if nk != nv:
        raise ValueError("k and v must have the same rows")
    _, _, qc, kc, _ = p._keep
    if qc is not None and (qc.shape[0] < nq or kc.shape[0] < nk):
        raise ValueError("the coordinates must have a row for each of their side's")
    return qp, ldq, nq, kp, ldk, vp, ldv, nk


def spv_attention(ws: Workspace, params: AttentionParams, q: torch.Tensor, k: torch.Tensor, v: torch.Tensor,
                  want_lse: bool = False, out: Optional[torch.Tensor] = None):
    """Attention of q [nq][H][D] over k, v [nk][Hkv][D] of the same scan; with want_lse (out, lse [nq][H])."""
    side = _qkv(params, q, k, v)
    nq, H, D = q.shape
    if out is None:
        out = torch.empty((nq, H, D), dtype=q.dtype, device=q.device)
    no, op, ldo = _heads(out, H, D, q.dtype, "out")
    if no != nq:
        raise ValueError("out must have q's rows")
    lse = torch.empty((nq, H), dtype=torch.float32, device=q.device) if want_lse else None
    st = lib().spv_attention(_stream(), ws.ptr, ws.nbytes, ct.byref(params), *side, op, ldo, _addr(lse), _DT[q.dtype])
    _chk(st, "spv_attention")
    return (out, lse) if want_lse else out


def spv_attention_backward(ws: Workspace, params: AttentionParams, q: torch.Tensor, k: torch.Tensor, v: torch.Tensor,
                           out: torch.Tensor, lse: torch.Tensor, dout: torch.Tensor,
                           grads: Optional[Sequence[torch.Tensor]] = None):
    """(dq, dk, dv) of spv_attention, given its out and lse [nq][H] and the gradient dout of out; grads: the
    tensors to write (which may be parts of one wider buffer), else new dense ones."""
    side = _qkv(params, q, k, v)
    nq, H, D = q.shape
    K, dt = params.Hkv, q.dtype
    no, op, ldo = _heads(out, H, D, dt, "out")
    nd, dop, lddo = _heads(dout, H, D, dt, "dout")
    if no != nq or nd != nq:
        raise ValueError("out and dout must have q's rows")
    if lse.dtype != torch.float32 or lse.shape != (nq, H):
        raise ValueError("lse must be float32 [rows][heads]")
    if grads is None:
        grads = [torch.empty(t.shape, dtype=dt, device=q.device) for t in (q, k, v)]
    elif any(g.shape[0] != t.shape[0] for g, t in zip(grads, (q, k, v))):
        raise ValueError("the gradients must have their inputs' rows")
    _, dq, lddq = _heads(grads[0], H, D, dt, "dq")
    _, dk, lddk = _heads(grads[1], K, D, dt, "dk")
    _, dv, lddv = _heads(grads[2], K, D, dt, "dv")
    st = lib().spv_attention_backward(_stream(), ws.ptr, ws.nbytes, ct.byref(params), *side, op, ldo, _addr(lse), dop,
                                      lddo, dq, lddq, dk, lddk, dv, lddv, _DT[dt])
    _chk(st, "spv_attention_backward")
    return tuple(grads)


def _here() -> int:
    """The current device, whose current stream the calls below run on: their tensors have to be there."""
    return torch.cuda.current_device()


def _stream_of(dev: int):
    return ct.c_void_p(_raw_stream(dev)) if _raw_stream is not None else _stream()


def _at(t: Optional[torch.Tensor], dev: int):
    """_addr of a tensor on device dev."""
    if t is None:
        return None
    if t.get_device() != dev:
        raise ValueError(f"libspv takes tensors of the current device, cuda:{dev}")
    if not t.is_contiguous():
        raise ValueError("libspv takes contiguous tensors")
    return t.data_ptr()


def _ws_at(ws: Workspace, dev: int):
    """Address of a workspace on device dev."""
    if ws.buf.get_device() != dev:
        raise ValueError(f"libspv takes a workspace of the current device, cuda:{dev}")
    return ws.ptr


def _vector(t: Optional[torch.Tensor], C: int, name: str, dev: int):
    """_channels of a tensor on device dev."""
    if t is not None and (t.dtype != torch.float32 or t.shape != (C,)):
        raise ValueError(f"{name} must be float32 [{C}]")
    return _at(t, dev)


def _count(t: Optional[torch.Tensor], dev: int):
    """Address of a device row count."""
    if t is not None and (t.dtype != torch.int64 or t.numel() < 1):
        raise ValueError("a row count is int64 [1]")
    return _at(t, dev)


def _rows_of(t: torch.Tensor, heads: int, D: int, dtype: torch.dtype, name: str, dev: int):
    """_heads of a tensor on device dev."""
    if t.get_device() != dev:
        raise ValueError(f"libspv takes tensors of the current device, cuda:{dev}")
    return _heads(t, heads, D, dtype, name)


def make_rope_params(D: int, freqs: torch.Tensor, sections: Sequence[int], halves: bool = False) -> RopeParams:
    """Parameters of a rotation of heads of D channels by voxel coordinates: sections = pairs of channels that turn
    with x, y and z; freqs [their sum] float32, radians a voxel.  Pair p is channels (2 p, 2 p + 1), or with halves
    (p, p + pairs).  The struct keeps a reference to freqs."""
    if len(sections) != 3:
        raise ValueError("sections are the pairs of x, y and z")
    p = RopeParams(D, (ct.c_int32 * 3)(*sections), int(halves), _channels(freqs, sum(sections), "freqs"))
    p._keep, p._ref = freqs, ct.byref(p)
    return p


def rope_freqs(sections: Sequence[int], longest: float = 100.0, device="cuda") -> torch.Tensor:
    """Radians a voxel of the pairs of each axis: from 1 down towards 1 / longest, evenly in their logarithms."""
    return torch.tensor([longest ** (-i / s) for s in sections for i in range(s)], dtype=torch.float32, device=device)


def spv_rope(params: RopeParams, coords: torch.Tensor, q: torch.Tensor, k: Optional[torch.Tensor] = None,
             inverse: bool = False, m_dev: Optional[torch.Tensor] = None,
             outs: Optional[Sequence[torch.Tensor]] = None):
    """q [n][H][D] (and k [n][Hkv][D]) rotated by the rows' coordinates [n][4]: q' or (q', k').  inverse: the
    rotation back, which turns gradients of the rotated rows into the rows'.  q, k and outs (the tensors to write, which
    may be q and k themselves) may be parts of wider rows."""
    D, dt, H, dev = params.D, q.dtype, q.shape[1], _here()
    n, qp, ldq = _rows_of(q, H, D, dt, "q", dev)
    kp = ko = None
    K = ldk = ldko = 0
    if k is not None:
        K = k.shape[1]
        nk, kp, ldk = _rows_of(k, K, D, dt, "k", dev)
        if nk != n:
            raise ValueError("q and k must have the same rows")
    if coords.dtype != torch.int32 or coords.dim() != 2 or coords.shape[1] != 4 or coords.shape[0] < n:
        raise ValueError(f"coords must be int32 [{n}][4]")
    if params._keep.get_device() != dev:
        raise ValueError(f"libspv takes tensors of the current device, cuda:{dev}")
    cp, count = _at(coords, dev), _count(m_dev, dev)
    if outs is None:
        outs = tuple(torch.empty_like(t, memory_format=torch.contiguous_format) for t in ((q,) if k is None else (q, k)))
        qo, ldqo = outs[0].data_ptr(), H * D
        if k is not None:
            ko, ldko = outs[1].data_ptr(), K * D
    else:
        sides = (q,) if k is None else (q, k)
        if len(outs) != len(sides) or any(o.shape != t.shape for o, t in zip(outs, sides)):
            raise ValueError("outs must have the shapes of what is rotated")
        _, qo, ldqo = _rows_of(outs[0], H, D, dt, "outs", dev)
        if k is not None:
            _, ko, ldko = _rows_of(outs[1], K, D, dt, "outs", dev)
    st = lib().spv_rope(_stream_of(dev), params._ref, cp, count, n, qp, ldq, H, kp, ldk, K, qo, ldqo, ko, ldko,
                        int(inverse), _DT[dt])
    _chk(st, "spv_rope")
    return outs[0] if k is None else tuple(outs)


@dataclass
class Checkpoint8:
    """Rows in 8 bits, as spv_checkpoint8 and spv_group_norm give them."""
    codes: torch.Tensor     # [m, C] int8
    exps: torch.Tensor      # [m, ceil(C / 32)] uint8
    dtype: torch.dtype      # of the rows they came from

    @classmethod
    def empty(cls, m: int, C: int, dtype: torch.dtype, device="cuda"):
        blocks = (C + SPV_CHECKPOINT8_BLOCK - 1) // SPV_CHECKPOINT8_BLOCK
        return cls(torch.empty((m, C), dtype=torch.int8, device=device),
                   torch.empty((m, blocks), dtype=torch.uint8, device=device), dtype)

    @classmethod
    def _like(cls, x: torch.Tensor):
        """A new one for rows like x, and its addresses."""
        m, C = x.shape
        codes = torch.empty_like(x, dtype=torch.int8, memory_format=torch.contiguous_format)
        exps = x.new_empty((m, (C + SPV_CHECKPOINT8_BLOCK - 1) // SPV_CHECKPOINT8_BLOCK), dtype=torch.uint8)
        return cls(codes, exps, x.dtype), codes.data_ptr(), exps.data_ptr()

    def addresses(self, dev: int):
        m, C = self.codes.shape
        if self.codes.dtype != torch.int8 or self.exps.dtype != torch.uint8 or \
                self.exps.shape != (m, (C + SPV_CHECKPOINT8_BLOCK - 1) // SPV_CHECKPOINT8_BLOCK):
            raise ValueError("a checkpoint is int8 [rows][channels] with uint8 [rows][blocks of 32 channels]")
        return _at(self.codes, dev), _at(self.exps, dev)


def spv_checkpoint8(x: torch.Tensor, m_dev: Optional[torch.Tensor] = None,
                    out: Optional[Checkpoint8] = None) -> Checkpoint8:
    """The rows x [m][C] in 8 bits, with an exponent for each 32 channels of a row."""
    m, C = x.shape
    dev = _here()
    xp, count = _at(x, dev), _count(m_dev, dev)
    if out is None:
        out, codes, exps = Checkpoint8._like(x)
    elif out.codes.shape != x.shape or out.dtype != x.dtype:
        raise ValueError("out must have x's shape and type")
    else:
        codes, exps = out.addresses(dev)
    st = lib().spv_checkpoint8(_stream_of(dev), xp, count, m, C, codes, exps, _DT[x.dtype])
    _chk(st, "spv_checkpoint8")
    return out


def spv_checkpoint8_read(saved: Checkpoint8, m_dev: Optional[torch.Tensor] = None,
                         out: Optional[torch.Tensor] = None) -> torch.Tensor:
    """The rows [m][C] that a checkpoint stands for, in the type they came from."""
    dev = _here()
    codes, exps = saved.addresses(dev)
    m, C = saved.codes.shape
    if out is None:
        out = torch.empty_like(saved.codes, dtype=saved.dtype)
    elif out.shape != (m, C) or out.dtype != saved.dtype:
        raise ValueError("out must have the rows' shape and type")
    op, count = _at(out, dev), _count(m_dev, dev)
    st = lib().spv_checkpoint8_read(_stream_of(dev), codes, exps, count, m, C, op, _DT[saved.dtype])
    _chk(st, "spv_checkpoint8_read")
    return out


def spv_linear_backward8(ws: Workspace, saved: Checkpoint8, da: torch.Tensor, m_dev: Optional[torch.Tensor] = None,
                         out: Optional[torch.Tensor] = None) -> torch.Tensor:
    """dW [Cin][Cout] float32 of a linear layer whose input rows were kept in 8 bits, given its product's gradient
    da [m][Cout]."""
    dev = _here()
    codes, exps = saved.addresses(dev)
    m, Cin = saved.codes.shape
    if da.dim() != 2 or da.shape[0] != m or da.dtype != saved.dtype:
        raise ValueError(f"da must be [{m}][Cout] of {saved.dtype}")
    Cout = da.shape[1]
    if out is None:
        out = da.new_empty((Cin, Cout), dtype=torch.float32)
    elif out.shape != (Cin, Cout) or out.dtype != torch.float32:
        raise ValueError(f"out must be float32 [{Cin}][{Cout}]")
    dap, op, count, wp = _at(da, dev), _at(out, dev), _count(m_dev, dev), _ws_at(ws, dev)
    st = lib().spv_linear_backward8(_stream_of(dev), wp, ws.nbytes, codes, exps, count, m, Cin, dap, Cout, op,
                                    _DT[da.dtype])
    _chk(st, "spv_linear_backward8")
    return out


def _scans(off: torch.Tensor) -> int:
    if off.dtype != torch.int32 or off.dim() != 1 or off.shape[0] < 1:
        raise ValueError("off must be int32 [scans + 1]")
    return off.shape[0] - 1


def spv_group_norm(ws: Workspace, x: torch.Tensor, off: torch.Tensor, groups: int,
                   gamma: Optional[torch.Tensor] = None, beta: Optional[torch.Tensor] = None, eps: float = 1e-5,
                   act: str = "none", want_stat: bool = False, want_checkpoint: bool = False,
                   out: Optional[torch.Tensor] = None):
    """act(group norm) of x [m][C] over the rows of each scan (off [scans + 1]) and the channels of each of `groups`
    groups; act is "none", "relu" or "silu".  y, or (y, stat), (y, checkpoint) or (y, stat, checkpoint): stat
    [scans][groups][2] and either x or its checkpoint in 8 bits are what the backward reads."""
    m, C = x.shape
    B = _scans(off)
    if act not in _ACT:
        raise ValueError(f"act must be one of {', '.join(_ACT)}")
    dev = _here()
    xp, gp, bp = _at(x, dev), _vector(gamma, C, "gamma", dev), _vector(beta, C, "beta", dev)
    if out is None:
        out = torch.empty_like(x)
    elif out.shape != x.shape or out.dtype != x.dtype:
        raise ValueError("out must have x's shape and type")
    offp, wp = _at(off, dev), _ws_at(ws, dev)
    stat = x.new_empty((B, groups, 2), dtype=torch.float32) if want_stat else None
    saved, codes, exps = Checkpoint8._like(x) if want_checkpoint else (None, None, None)
    st = lib().spv_group_norm(_stream_of(dev), wp, ws.nbytes, xp, m, C, offp, B, groups, gp, bp, eps, _ACT[act],
                              _at(out, dev), _at(stat, dev), codes, exps, _DT[x.dtype])
    _chk(st, "spv_group_norm")
    got = (out, *(t for t in (stat, saved) if t is not None))
    return got if len(got) > 1 else out


def spv_group_norm_backward(ws: Workspace, dy: torch.Tensor, x, off: torch.Tensor, groups: int, stat: torch.Tensor,
                            gamma: Optional[torch.Tensor] = None, beta: Optional[torch.Tensor] = None,
                            act: str = "none", dres: Optional[torch.Tensor] = None):
    """(dx, dgamma, dbeta) of spv_group_norm, given its stat and x or x's checkpoint; dres: a gradient added to dx (the
    residual branch's)."""
    m, C = dy.shape
    B = _scans(off)
    if act not in _ACT:
        raise ValueError(f"act must be one of {', '.join(_ACT)}")
    dev = _here()
    codes = exps = xp = None
    if isinstance(x, Checkpoint8):
        if x.codes.shape != dy.shape or x.dtype != dy.dtype:
            raise ValueError("the checkpoint must have dy's shape and type")
        codes, exps = x.addresses(dev)
    else:
        if x.shape != dy.shape or x.dtype != dy.dtype:
            raise ValueError("x must have dy's shape and type")
        xp = _at(x, dev)
    if dres is not None and (dres.shape != dy.shape or dres.dtype != dy.dtype):
        raise ValueError("dres must have dy's shape and type")
    if stat.dtype != torch.float32 or stat.shape != (B, groups, 2):
        raise ValueError(f"stat must be float32 [{B}][{groups}][2]")
    dyp, offp, sp, rp = _at(dy, dev), _at(off, dev), _at(stat, dev), _at(dres, dev)
    gp, bp, wp = _vector(gamma, C, "gamma", dev), _vector(beta, C, "beta", dev), _ws_at(ws, dev)
    dx = torch.empty_like(dy)
    dgamma = dy.new_empty(C, dtype=torch.float32)
    dbeta = torch.empty_like(dgamma)
    st = lib().spv_group_norm_backward(_stream_of(dev), wp, ws.nbytes, dyp, xp, codes, exps, m, C, offp, B, groups, gp,
                                       bp, sp, _ACT[act], rp, dx.data_ptr(), dgamma.data_ptr(), dbeta.data_ptr(),
                                       _DT[dy.dtype])
    _chk(st, "spv_group_norm_backward")
    return dx, dgamma, dbeta


def spv_devoxelize(ws: Workspace, grid_coords: torch.Tensor, vfeat: torch.Tensor, xyz: torch.Tensor,
                   voxel_size: float, stride_log2: int = 0, mode: int = SPV_DEVOX_CENTER,
                   batch: Optional[torch.Tensor] = None, m_dev: Optional[torch.Tensor] = None,
                   m_cap: Optional[int] = None, pfeat: Optional[torch.Tensor] = None, Wp: Optional[torch.Tensor] = None,
                   scale_p: Optional[torch.Tensor] = None, shift_p: Optional[torch.Tensor] = None,
                   relu_p: bool = False, want_corners: bool = False, out: Optional[torch.Tensor] = None):
    n = xyz.shape[0]
    C = vfeat.shape[1]
    m_cap = grid_coords.shape[0] if m_cap is None else m_cap
    Cp = pfeat.shape[1] if pfeat is not None else 0
    if out is None:
        out = torch.empty((max(n, 1), C), dtype=vfeat.dtype, device=xyz.device)
    ci = torch.empty((max(n, 1), 8), dtype=torch.int32, device=xyz.device) if want_corners else None
    cw = torch.empty((max(n, 1), 8), dtype=torch.float32, device=xyz.device) if want_corners else None
    st = lib().spv_devoxelize(_stream(), ws.ptr, ws.nbytes, _ptr(grid_coords), _ptr(m_dev), m_cap, stride_log2,
                              _ptr(xyz), _ptr(batch), n, ct.c_float(voxel_size), mode, _ptr(vfeat), C, _ptr(pfeat),
                              Cp, _ptr(Wp), _ptr(scale_p), _ptr(shift_p), int(relu_p), _ptr(out), _DT[vfeat.dtype],
                              _ptr(ci), _ptr(cw))
    _chk(st, "spv_devoxelize")
    return (out, ci, cw) if want_corners else out


def spv_devoxelize_nbr(ws: Workspace, grid_coords: torch.Tensor, vfeat: torch.Tensor, nbr: torch.Tensor,
                       pt2vox: torch.Tensor, xyz: torch.Tensor, voxel_size: float, stride_log2: int = 0,
                       mode: int = SPV_DEVOX_CENTER, batch: Optional[torch.Tensor] = None,
                       m_dev: Optional[torch.Tensor] = None, m_cap: Optional[int] = None,
                       pfeat: Optional[torch.Tensor] = None, Wp: Optional[torch.Tensor] = None,
                       scale_p: Optional[torch.Tensor] = None, shift_p: Optional[torch.Tensor] = None,
                       relu_p: bool = False, out: Optional[torch.Tensor] = None) -> torch.Tensor:
    """spv_devoxelize on the points' own voxelization at that stride: corners from the neighbour table."""
    n = xyz.shape[0]
    C = vfeat.shape[1]
    m_cap = grid_coords.shape[0] if m_cap is None else m_cap
    Cp = pfeat.shape[1] if pfeat is not None else 0
    if out is None:
        out = torch.empty((max(n, 1), C), dtype=vfeat.dtype, device=xyz.device)
    st = lib().spv_devoxelize_nbr(_stream(), ws.ptr, ws.nbytes, _ptr(grid_coords), _ptr(m_dev), m_cap, _ptr(nbr),
                                  _ptr(pt2vox), stride_log2, _ptr(xyz), _ptr(batch), n, ct.c_float(voxel_size), mode,
                                  _ptr(vfeat), C, _ptr(pfeat), Cp, _ptr(Wp), _ptr(scale_p), _ptr(shift_p), int(relu_p),
                                  _ptr(out), _DT[vfeat.dtype])
    _chk(st, "spv_devoxelize_nbr")
    return out


def make_block_params(C: int, dtype: torch.dtype, voxel_size: float, convs: Sequence, Wp: torch.Tensor,
                      scale_p=None, shift_p=None, relu_p: bool = True, mode: int = SPV_DEVOX_CENTER,
                      residual: bool = False) -> BlockParams:
    """convs: list of (W [27,C,C], scale|None, shift|None, relu) device tensors.

    The struct holds raw device pointers; it also keeps references to every
    tensor it points into, so they stay allocated as long as the struct lives."""
    def ptr(t):
        return None if t is None else _ptr(t).value
    p = BlockParams()
    p.C, p.dtype, p.voxel_size, p.n_convs = C, _DT[dtype], voxel_size, len(convs)
    keep = [Wp, scale_p, shift_p]
    for l, (W, sc, sh, r) in enumerate(convs):
        p.W[l] = ptr(W)
        p.scale[l] = ptr(sc)
        p.shift[l] = ptr(sh)
        p.relu[l] = int(r)
        keep += [W, sc, sh]
    p.Wp = ptr(Wp)
    p.scale_p = ptr(scale_p)
    p.shift_p = ptr(shift_p)
    p.relu_p = int(relu_p)
    p.devox_mode = mode
    p.residual = int(residual)
    p._keep = keep
    return p


def spv_block(ws: Workspace, params: BlockParams, xyz: torch.Tensor, feat: torch.Tensor,
              batch: Optional[torch.Tensor] = None, out: Optional[torch.Tensor] = None, sync: bool = False):
    n, C = feat.shape
    if out is None:
        out = torch.empty((max(n, 1), C), dtype=feat.dtype, device=feat.device)
    m = ct.c_int64(0)
    st = lib().spv_block(_stream(), ws.ptr, ws.nbytes, ct.byref(params), _ptr(xyz), _ptr(batch), n, _ptr(feat),
                         _ptr(out), ct.byref(m) if sync else None)
    _chk(st, "spv_block")
    return (out, m.value) if sync else out


def spv_lookup(ws: Workspace, table_coords: torch.Tensor, qcoords: torch.Tensor,
               m_dev: Optional[torch.Tensor] = None) -> torch.Tensor:
    q = qcoords.shape[0]
    idx = torch.empty(max(q, 1), dtype=torch.int32, device=qcoords.device)
    st = lib().spv_lookup(_stream(), ws.ptr, ws.nbytes, _ptr(table_coords), _ptr(m_dev), table_coords.shape[0],
                          _ptr(qcoords), q, _ptr(idx))
    _chk(st, "spv_lookup")
    return idx[:q]


def spv_voxel_lookup(ws: Workspace, n: int, qcoords: torch.Tensor) -> torch.Tensor:
    """Lookups in the table the last spv_voxelize(ws, ..., n points) built."""
    q = qcoords.shape[0]
    idx = torch.empty(max(q, 1), dtype=torch.int32, device=qcoords.device)
    st = lib().spv_voxel_lookup(_stream(), ws.ptr, ws.nbytes, n, _ptr(qcoords), q, _ptr(idx))
    _chk(st, "spv_voxel_lookup")
    return idx[:q]


def spv_conv_kernel(K3: int, Cin: int, Cout: int, dtype: torch.dtype, in_rows: int, m_out_cap: int,
                    pair_cap: int, transposed: bool = False) -> int:
    """Host query: 0 neighbour-table MFMA on 27 offsets, 1 MFMA on a table of 8 or on tiles of pairs,
    2 float32 rows, -1 rejected."""
    return lib().spv_conv_kernel(K3, Cin, Cout, _DT[dtype], in_rows, m_out_cap, pair_cap, int(transposed))


def spv_block_conv_kernel(n: int, C: int, dtype: torch.dtype) -> int:
    return lib().spv_block_conv_kernel(n, C, _DT[dtype])
