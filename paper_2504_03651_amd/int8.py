"""Python binding of the linear layers in 8-bit integers (include/echo_int8.h): checks
of the tensors, then the library's calls on PyTorch's current stream.

Codes are tensors of torch.int8, scales fp32, one a row: [T] for activations [T][K],
[N] for weights [N][K].
"""
from __future__ import annotations

import ctypes

from . import echo, fp8
from .fp8 import BF16, F32, address, refuse, rows, scratch, sizes, stream_of

SYMBOLS = ["echo_int8_quantize", "echo_int8_gemm", "echo_int8_gemm_workspace_bytes"]

_bound = False
_codes = None


def _lib():
    global _bound, _codes
    L = echo.lib()
    if not _bound:
        import torch
        vp, i32, i64, sz = ctypes.c_void_p, ctypes.c_int32, ctypes.c_int64, ctypes.c_size_t
        L.echo_int8_quantize.argtypes = [vp, i32, i64, i32, i32, vp, vp, vp]
        L.echo_int8_quantize.restype = ctypes.c_int
        L.echo_int8_gemm_workspace_bytes.argtypes = [i32, i32, i32]
        L.echo_int8_gemm_workspace_bytes.restype = sz
        L.echo_int8_gemm.argtypes = [vp, vp, vp, vp, i32, i32, i32, vp, vp, vp, i32, i64, vp, sz, vp]
        L.echo_int8_gemm.restype = ctypes.c_int
        _codes = (torch.int8,)
        _bound = True
    return L


def quantize(x, codes, scales, stream=None) -> None:
    """Codes and scales of the rows of ``x`` [rows][cols] (any distance apart), bf16 or
    fp32."""
    where, k, L = "echo_int8_quantize", fp8.types(), _lib()
    dev = k.device()
    shape = x.shape
    if len(shape) != 2:
        refuse(where, f"x has {x.dim()} axes")
    n, cols = shape
    if (n | cols) >> 31:
        sizes(where, n, cols)
    xp, stride = rows(where, "x", x, shape, k.real, dev)
    cp = address(where, "codes", codes, shape, _codes, dev)
    sp = address(where, "scales", scales, (n,), k.f32, dev)
    rc = L.echo_int8_quantize(xp, F32 if x.dtype is k.f32[0] else BF16, stride, n, cols, cp, sp,
                              stream_of(stream, dev))
    if rc:
        echo._check(rc, where)


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
    where, k, L = "echo_int8_gemm", fp8.types(), _lib()
    dev = k.device()
    if x.dim() != 2 or w.dim() != 2:
        refuse(where, f"x has {x.dim()} axes, w {w.dim()}")
    (T, K), N = x.shape, w.shape[0]
    if (T | K | N) >> 31:
        sizes(where, T, K, N)
    xp = address(where, "x", x, (T, K), _codes, dev)
    xsp = address(where, "x_scale", x_scale, (T,), k.f32, dev)
    wp = address(where, "w", w, (N, K), _codes, dev)
    wsp = address(where, "w_scale", w_scale, (N,), k.f32, dev)
    yp, stride = rows(where, "out", out, (T, N), k.real, dev)
    bp = None if bias is None else address(where, "bias", bias, (N,), k.f32, dev)
    rp = None
    if residual is not None:
        rp, rs = rows(where, "residual", residual, (T, N), k.real, dev)
        if residual.dtype is not out.dtype or rs != stride:
            refuse(where, "residual has not the type and strides of out")
    sp, sb = scratch(where, workspace, dev)
    rc = L.echo_int8_gemm(xp, xsp, wp, wsp, T, N, K, bp, rp, yp, F32 if out.dtype is k.f32[0] else BF16,
                          stride, sp, sb, stream_of(stream, dev))
    if rc:
        echo._check(rc, where)
