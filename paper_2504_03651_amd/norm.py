"""Python binding of the norms between blocks (include/echo_norm.h): checks of the
tensors, then the library's calls on PyTorch's current stream."""
from __future__ import annotations

import ctypes

from . import echo, fp8
from .fp8 import BF16, F32, address, refuse, rows, sizes, stream_of

SYMBOLS = ["echo_norm_join"]

KINDS = {"none": 0, "rms": 1, "layer": 2}
I8 = 2


class CNorm(ctypes.Structure):
    _fields_ = [*[(n, ctypes.c_int32) for n in ("hidden", "post", "pre", "param_dtype")],
                *[(n, ctypes.c_float) for n in ("post_eps", "pre_eps", "residual_scale", "block_scale",
                                                "weight_offset")],
                *[(n, ctypes.c_void_p) for n in ("post_weight", "post_bias", "pre_weight", "pre_bias")]]


class CRows(ctypes.Structure):
    _fields_ = [("data", ctypes.c_void_p), ("dtype", ctypes.c_int32), ("stride", ctypes.c_int64)]


_bound = False
_dtypes = {}
_out = ()


def _lib():
    global _bound, _out
    L = echo.lib()
    if not _bound:
        import torch
        vp, i32 = ctypes.c_void_p, ctypes.c_int32
        R = ctypes.POINTER(CRows)
        L.echo_norm_join.argtypes = [ctypes.POINTER(CNorm), i32, R, R, R, R, R, vp, vp]
        L.echo_norm_join.restype = ctypes.c_int
        _dtypes.update({torch.bfloat16: BF16, torch.float32: F32, torch.int8: I8})
        _out = (torch.bfloat16, torch.float32, torch.int8)
        _bound = True
    return L


class Norm:
    """The norms ``post`` (behind a block) and ``pre`` (before the next), each "none",
    "rms" or "layer", and the scales of residual and block (echo_norm_t).  Weights and
    biases [hidden] are bf16 or fp32, all alike, or None: 1 and 0."""

    def __init__(self, hidden: int, post: str = "none", pre: str = "none", post_weight=None,
                 post_bias=None, pre_weight=None, pre_bias=None, post_eps: float = 1e-5,
                 pre_eps: float = 1e-5, residual_scale: float = 1.0, block_scale: float = 1.0,
                 weight_offset: float = 0.0):
        where, k = "Norm", fp8.types()
        for kind in (post, pre):
            if kind not in KINDS:
                raise echo.EchoError(echo.ECHO_E_UNSUPPORTED, where, f"norm {kind!r}")
        sizes(where, hidden)
        self.t = (post_weight, post_bias, pre_weight, pre_bias)   # kept alive
        given = [t for t in self.t if t is not None]
        self.device = given[0].get_device() if given else None
        if self.device is not None and self.device < 0:
            refuse(where, "the weights are not on a GPU")
        dtypes = (given[0].dtype,) if given else k.real
        if dtypes[0] not in k.real:
            refuse(where, f"weights have dtype {dtypes[0]}")
        at = [None if t is None else address(where, n, t, (hidden,), dtypes, self.device)
              for n, t in zip(("post_weight", "post_bias", "pre_weight", "pre_bias"), self.t)]
        _lib()
        self.hidden = hidden
        self.c = CNorm(hidden, KINDS[post], KINDS[pre], _dtypes[dtypes[0]], post_eps, pre_eps,
                       residual_scale, block_scale, weight_offset, *at)
        self.ref = ctypes.byref(self.c)


def _rows(where, name, t, shape, dtypes, dev):
    if t is None:
        return None
    p, stride = rows(where, name, t, shape, dtypes, dev)
    return ctypes.byref(CRows(p, _dtypes[t.dtype], stride))


def join(norm: Norm, block, residual, gate=None, sum=None, y=None, y_scale=None, stream=None) -> None:
    """sum = residual_scale * residual + block_scale * gate * post(block), y = pre(sum).

    Rows [T][hidden] (any distance apart), bf16 or fp32, each of a type of its own; block
    or residual may be None, gate (also [hidden]: one row for every token) 1, sum or y
    not wanted.  y may be int8 codes with scales ``y_scale`` fp32 [T]."""
    where, k, L = "echo_norm_join", fp8.types(), _lib()
    dev = k.device()
    if norm.device is not None and norm.device != dev:
        refuse(where, f"the weights are on cuda:{norm.device}, the current device is cuda:{dev}")
    lead = block if block is not None else residual
    if lead is None:
        refuse(where, "neither block nor residual")
    if lead.dim() != 2:
        refuse(where, f"block or residual has {lead.dim()} axes")
    T, H = lead.shape[0], norm.hidden
    if T >> 31:
        sizes(where, T)
    shape = (T, H)
    if gate is not None and gate.dim() == 1:
        gp = address(where, "gate", gate, (H,), k.real, dev)
        gr = ctypes.byref(CRows(gp, _dtypes[gate.dtype], 0))
    else:
        gr = _rows(where, "gate", gate, shape, k.real, dev)
    br = _rows(where, "block", block, shape, k.real, dev)
    rr = _rows(where, "residual", residual, shape, k.real, dev)
    sr = _rows(where, "sum", sum, shape, k.real, dev)
    yr = _rows(where, "y", y, shape, _out, dev)
    sp = None
    if y_scale is not None:
        sp = address(where, "y_scale", y_scale, (T,), k.f32, dev)
    rc = L.echo_norm_join(norm.ref, T, br, gr, rr, sr, yr, sp, stream_of(stream, dev))
    if rc:
        echo._check(rc, where)
