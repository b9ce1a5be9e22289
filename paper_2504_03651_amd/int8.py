"""Python binding of the linear layers in 8-bit integers (include/echo_int8.h): checks
of the tensors, then the library's calls on PyTorch's current stream.

Codes are tensors of torch.int8, scales fp32, one a row: [T] for activations [T][K],
[N] for weights [N][K].
"""
from __future__ import annotations

import ctypes

from . import echo, native
from .fp8 import sizes

SYMBOLS = ["echo_int8_quantize", "echo_int8_gemm", "echo_int8_gemm_workspace_bytes"]

_bound = False


def _lib():
    global _bound
    L = echo.lib()
    if not _bound:
        vp, i32, i64, sz = ctypes.c_void_p, ctypes.c_int32, ctypes.c_int64, ctypes.c_size_t
        L.echo_int8_quantize.argtypes = [vp, i32, i64, i32, i32, vp, vp, vp]
        L.echo_int8_quantize.restype = ctypes.c_int
        L.echo_int8_gemm_workspace_bytes.argtypes = [i32, i32, i32]
        L.echo_int8_gemm_workspace_bytes.restype = sz
        L.echo_int8_gemm.argtypes = [vp, vp, vp, vp, i32, i32, i32, vp, vp, vp, i32, i64, vp, sz, vp]
        L.echo_int8_gemm.restype = ctypes.c_int
        _bound = True
    return L


def quantize(x, codes, scales, stream=None) -> None:
    """Codes and scales of the rows of ``x`` [rows][cols] (any distance apart), bf16 or
    fp32."""
    native.binding().quantize(x, codes, scales, stream)


def gemm_workspace_bytes(num_tokens: int, out_features: int, in_features: int) -> int:
    """Enough for every product of up to ``num_tokens`` tokens with such weights."""
    where = "echo_int8_gemm_workspace_bytes"
    sizes(where, num_tokens, out_features, in_features)
    n = int(_lib().echo_int8_gemm_workspace_bytes(int(num_tokens), int(out_features), int(in_features)))
    if n == 0 and echo.last_error():
        raise echo.EchoError(echo.ECHO_E_INVALID, where, echo.last_error())
    return n


def gemm(x, x_scale, w, w_scale, out, bias=None, residual=None, workspace=None, stream=None) -> None:
    """out [T][N] (bf16 or fp32, rows any distance apart) = x [T][K] times the
    transpose of w [N][K], plus ``bias`` (fp32 [N]), plus ``residual`` (of out's type and
    strides; may be out itself).  ``workspace``: gemm_workspace_bytes() bytes, None
    where that is 0."""
    native.binding().gemm(x, x_scale, w, w_scale, out, bias, residual, workspace, stream)
