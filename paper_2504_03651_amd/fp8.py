"""Python binding of the 8-bit linear layers (include/echo_fp8.h): checks of the
tensors, then the library's calls on PyTorch's current stream.

Codes are tensors of torch.float8_e4m3fn (or their bytes, torch.uint8), scales
fp32: a matrix [rows][cols] has scales [ceil(rows / block_rows)][ceil(cols / 128)].
"""
from __future__ import annotations

import ctypes

from . import echo

SYMBOLS = ["echo_fp8_quantize", "echo_fp8_gemm", "echo_fp8_gemm_workspace_bytes"]

BLOCK = 128
BF16, F32 = 0, 1

_bound = False


def _lib():
    global _bound
    L = echo.lib()
    if not _bound:
        vp, i32, i64, sz = ctypes.c_void_p, ctypes.c_int32, ctypes.c_int64, ctypes.c_size_t
        L.echo_fp8_quantize.argtypes = [vp, i32, i64, i32, i32, i32, i32, vp, vp, vp]
        L.echo_fp8_quantize.restype = ctypes.c_int
        L.echo_fp8_gemm_workspace_bytes.argtypes = [i32, i32, i32]
        L.echo_fp8_gemm_workspace_bytes.restype = sz
        L.echo_fp8_gemm.argtypes = [vp, vp, vp, vp, i32, i32, i32, vp, vp, i32, i64, vp, sz, vp]
        L.echo_fp8_gemm.restype = ctypes.c_int
        _bound = True
    return L


def blocks(n: int) -> int:
    """Scales along an axis of n values."""
    return -(-n // BLOCK)


def _refuse(where: str, what: str):
    raise echo.EchoError(echo.ECHO_E_INVALID, where, what)


_dtypes = {}


def _kinds():
    if not _dtypes:
        import torch
        _dtypes.update(codes=(torch.float8_e4m3fn, torch.uint8), f32=(torch.float32,),
                       bf16=(torch.bfloat16,), i32=(torch.int32,),
                       real=(torch.bfloat16, torch.float32))
    return _dtypes


def check(where: str, name: str, t, shape, kind: str, rows: bool = False) -> None:
    """Refuses a tensor of another shape, type, device or layout: contiguous, or
    with ``rows`` of contiguous rows any distance apart."""
    if tuple(t.shape) != tuple(shape):
        _refuse(where, f"{name} has shape {tuple(t.shape)}, not {tuple(shape)}")
    if t.dtype not in _kinds()[kind]:
        _refuse(where, f"{name} has dtype {t.dtype}")
    on_device(where, name, t)
    if rows:
        if t.numel() and (t.stride(-1) != 1 and t.shape[-1] > 1 or
                          t.shape[0] > 1 and t.stride(0) < t.shape[-1]):
            _refuse(where, f"the rows of {name} are not contiguous")
    elif not t.is_contiguous():
        _refuse(where, f"{name} is not contiguous")


def on_device(where: str, name: str, t) -> None:
    import torch
    if t.device.type != "cuda":
        _refuse(where, f"{name} is on {t.device}, not on a GPU")
    if t.device.index != torch.cuda.current_device():
        _refuse(where, f"{name} is on {t.device}, the current device is "
                       f"cuda:{torch.cuda.current_device()}")


def row_stride(t) -> int:
    return max(t.stride(0), t.shape[-1]) if t.shape[0] > 1 else max(1, t.shape[-1])


def real_dtype(t) -> int:
    import torch
    return F32 if t.dtype is torch.float32 else BF16


def _workspace(where: str, t):
    """(pointer, bytes) of a workspace tensor or None."""
    if t is None:
        return None, 0
    on_device(where, "workspace", t)
    if not t.is_contiguous():
        _refuse(where, "workspace is not contiguous")
    return t.data_ptr(), t.numel() * t.element_size()


def quantize(x, codes, scales, block_rows: int = 1, stream=None) -> None:
    """Codes and scales of ``x`` [rows][cols] (rows any distance apart) or
    [batch][rows][cols], bf16 or fp32, in blocks of ``block_rows`` (1 or 128) x 128."""
    where = "echo_fp8_quantize"
    if x.dim() not in (2, 3):
        _refuse(where, f"x has {x.dim()} axes")
    if block_rows not in (1, BLOCK):
        raise echo.EchoError(echo.ECHO_E_UNSUPPORTED, where, f"block_rows {block_rows}")
    rows, cols = x.shape[-2:]
    check(where, "x", x, x.shape, "real", rows=x.dim() == 2)
    check(where, "codes", codes, x.shape, "codes")
    check(where, "scales", scales, (*x.shape[:-2], -(-rows // block_rows), blocks(cols)), "f32")
    batch = x.shape[0] if x.dim() == 3 else 1
    echo._check(_lib().echo_fp8_quantize(
        x.data_ptr(), real_dtype(x), row_stride(x) if x.dim() == 2 else cols, batch, rows, cols,
        block_rows, codes.data_ptr(), scales.data_ptr(), echo._stream(stream)), where)


def gemm_workspace_bytes(num_tokens: int, out_features: int, in_features: int) -> int:
    n = int(_lib().echo_fp8_gemm_workspace_bytes(int(num_tokens), int(out_features),
                                                 int(in_features)))
    if n == 0 and echo.last_error():
        raise echo.EchoError(echo.ECHO_E_INVALID, "echo_fp8_gemm_workspace_bytes",
                             echo.last_error())
    return n


def gemm(x, x_scale, w, w_scale, out, residual=None, workspace=None, stream=None) -> None:
    """out [T][N] (bf16 or fp32, rows any distance apart) = x [T][K] times the
    transpose of w [N][K], plus ``residual`` (of out's type and strides; may be
    out itself).  ``workspace``: gemm_workspace_bytes() bytes, None where that is 0."""
    where = "echo_fp8_gemm"
    if x.dim() != 2 or w.dim() != 2:
        _refuse(where, f"x has {x.dim()} axes, w {w.dim()}")
    (T, K), N = x.shape, w.shape[0]
    check(where, "x", x, (T, K), "codes")
    check(where, "x_scale", x_scale, (T, blocks(K)), "f32")
    check(where, "w", w, (N, K), "codes")
    check(where, "w_scale", w_scale, (blocks(N), blocks(K)), "f32")
    check(where, "out", out, (T, N), "real", rows=True)
    if residual is not None:
        check(where, "residual", residual, (T, N), "real", rows=True)
        if residual.dtype is not out.dtype or row_stride(residual) != row_stride(out):
            _refuse(where, "residual has not the type and strides of out")
    wp, wb = _workspace(where, workspace)
    echo._check(_lib().echo_fp8_gemm(
        x.data_ptr(), x_scale.data_ptr(), w.data_ptr(), w_scale.data_ptr(), T, N, K,
        None if residual is None else residual.data_ptr(), out.data_ptr(), real_dtype(out),
        row_stride(out), wp, wb, echo._stream(stream)), where)
