"""Python binding of the norms between blocks (include/echo_norm.h): checks of the
tensors, then the library's calls on PyTorch's current stream."""
from __future__ import annotations

import ctypes

from . import echo, fp8, native
from .fp8 import BF16, F32, address, refuse, sizes

SYMBOLS = ["echo_norm_join"]

KINDS = {"none": 0, "rms": 1, "layer": 2}


class CNorm(ctypes.Structure):
    _fields_ = [*[(n, ctypes.c_int32) for n in ("hidden", "post", "pre", "param_dtype")],
                *[(n, ctypes.c_float) for n in ("post_eps", "pre_eps", "residual_scale", "block_scale",
                                                "weight_offset")],
                *[(n, ctypes.c_void_p) for n in ("post_weight", "post_bias", "pre_weight", "pre_bias")]]


class CRows(ctypes.Structure):
    _fields_ = [("data", ctypes.c_void_p), ("dtype", ctypes.c_int32), ("stride", ctypes.c_int64)]


_bound = False


def _lib():
    global _bound
    L = echo.lib()
    if not _bound:
        vp, i32 = ctypes.c_void_p, ctypes.c_int32
        R = ctypes.POINTER(CRows)
        L.echo_norm_join.argtypes = [ctypes.POINTER(CNorm), i32, R, R, R, R, R, vp, vp]
        L.echo_norm_join.restype = ctypes.c_int
        _bound = True
    return L


class Norm:
    """The norms ``post`` (behind a block) and ``pre`` (before the next), each "none",
    "rms" or "layer", and the scales of residual and block (echo_norm_t).  Weights and
    biases [hidden] are bf16 or fp32, all alike, or None: 1 and 0.  They are read at each
    call, in the memory that they have now."""

    def __init__(self, hidden: int, post: str = "none", pre: str = "none", post_weight=None,
                 post_bias=None, pre_weight=None, pre_bias=None, post_eps: float = 1e-5,
                 pre_eps: float = 1e-5, residual_scale: float = 1.0, block_scale: float = 1.0,
                 weight_offset: float = 0.0):
        where, k = "Norm", fp8.types()
        for kind in (post, pre):
            if kind not in KINDS:
                raise echo.EchoError(echo.ECHO_E_UNSUPPORTED, where, f"norm {kind!r}")
        sizes(where, hidden)
        # kept alive, also where a parameter is given another tensor later
        self.t = tuple(t if t is None else t.detach() for t in (post_weight, post_bias, pre_weight, pre_bias))
        given = [t for t in self.t if t is not None]
        self.device = given[0].get_device() if given else None
        if self.device is not None and self.device < 0:
            refuse(where, "the weights are not on a GPU")
        dtypes = (given[0].dtype,) if given else k.real
        if dtypes[0] not in k.real:
            refuse(where, f"weights have dtype {dtypes[0]}")
        at = [None if t is None else address(where, n, t, (hidden,), dtypes, self.device)
              for n, t in zip(("post_weight", "post_bias", "pre_weight", "pre_bias"), self.t)]
        self.hidden = hidden
        self.c = CNorm(hidden, KINDS[post], KINDS[pre], F32 if dtypes[0] is k.f32[0] else BF16, post_eps, pre_eps,
                       residual_scale, block_scale, weight_offset, *at)
        self.at = ctypes.addressof(self.c)


def join(norm: Norm, block, residual, gate=None, sum=None, y=None, y_scale=None, stream=None) -> None:
    """sum = residual_scale * residual + block_scale * gate * post(block), y = pre(sum).

    Rows [T][hidden] (any distance apart), bf16 or fp32, each of a type of its own; block
    or residual may be None, gate (also [hidden]: one row for every token) 1, sum or y
    not wanted.  y may be int8 codes with scales ``y_scale`` fp32 [T]."""
    native.binding().join(norm.at, norm.device, block, residual, gate, sum, y, y_scale, stream)
