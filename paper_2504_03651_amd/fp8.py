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


def refuse(where: str, what: str):
    raise echo.EchoError(echo.ECHO_E_INVALID, where, what)


def sizes(where: str, *n: int):
    """Refuses counts that the library's 32-bit arguments would cut off."""
    for v in n:
        if not -2 ** 31 <= v < 2 ** 31:
            refuse(where, f"{v} is not below 2^31")


class _Types:
    """Types that tensors may have (filled in at the first call: importing this
    module does not import torch)."""
    codes = f32 = bf16 = i32 = real = device = raw_stream = None


def types():
    if _Types.real is None:
        import torch
        _Types.codes, _Types.f32 = (torch.float8_e4m3fn, torch.uint8), (torch.float32,)
        _Types.bf16, _Types.i32 = (torch.bfloat16,), (torch.int32,)
        # no GPU: a device that no tensor is on
        _Types.device = torch.cuda.current_device if torch.cuda.is_available() else lambda: -2
        _Types.raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None)
        _Types.real = (torch.bfloat16, torch.float32)
    return _Types


def _place(where: str, name: str, t, dev: int):
    refuse(where, f"{name} is on {t.device}, " + (f"the current device is cuda:{dev}" if t.is_cuda
                                                  else "not on a GPU"))


def address(where: str, name: str, t, shape, dtypes, dev: int) -> int:
    """The address of a contiguous tensor of this shape, one of these types, on
    the current device; refuses any other."""
    if t.shape != shape:
        refuse(where, f"{name} has shape {tuple(t.shape)}, not {tuple(shape)}")
    if t.dtype not in dtypes:
        refuse(where, f"{name} has dtype {t.dtype}")
    if t.get_device() != dev:
        _place(where, name, t, dev)
    if not t.is_contiguous():
        refuse(where, f"{name} is not contiguous")
    return t.data_ptr()


def rows(where: str, name: str, t, shape, dtypes, dev: int):
    """(address, elements from row to row) of a matrix whose rows are contiguous
    and any distance apart."""
    if t.shape != shape:
        refuse(where, f"{name} has shape {tuple(t.shape)}, not {tuple(shape)}")
    if t.dtype not in dtypes:
        refuse(where, f"{name} has dtype {t.dtype}")
    if t.get_device() != dev:
        _place(where, name, t, dev)
    n, m = shape
    if t.is_contiguous():
        return t.data_ptr(), max(m, 1)
    s, one = t.stride()
    if m > 1 and one != 1 or n > 1 and s < m:
        refuse(where, f"the rows of {name} are not contiguous")
    return t.data_ptr(), s if n > 1 else max(m, 1)


def scratch(where: str, t, dev: int):
    """(address, bytes) of a workspace tensor or None."""
    if t is None:
        return None, 0
    if t.get_device() != dev:
        _place(where, "workspace", t, dev)
    if not t.is_contiguous():
        refuse(where, "workspace is not contiguous")
    return t.data_ptr(), t.nbytes


def stream_of(stream, dev: int) -> int:
    return types().raw_stream(dev) if stream is None else stream.cuda_stream


def quantize(x, codes, scales, block_rows: int = 1, stream=None) -> None:
    """Codes and scales of ``x`` [rows][cols] (rows any distance apart) or
    [batch][rows][cols], bf16 or fp32, in blocks of ``block_rows`` (1 or 128) x 128."""
    where, k = "echo_fp8_quantize", types()
    dev = k.device()
    shape = x.shape
    if block_rows != 1 and block_rows != BLOCK:
        raise echo.EchoError(echo.ECHO_E_UNSUPPORTED, where, f"block_rows {block_rows}")
    if len(shape) == 2:
        batch, (n, cols), lead = 1, shape, ()
        if (n | cols) >> 31:
            sizes(where, n, cols)
        xp, stride = rows(where, "x", x, shape, k.real, dev)
    elif len(shape) == 3:
        batch, n, cols = shape
        if (batch | n | cols) >> 31:
            sizes(where, batch, n, cols)
        xp, stride, lead = address(where, "x", x, shape, k.real, dev), cols, (batch,)
    else:
        refuse(where, f"x has {x.dim()} axes")
    cp = address(where, "codes", codes, shape, k.codes, dev)
    sp = address(where, "scales", scales, (*lead, -(-n // block_rows), -(-cols // BLOCK)), k.f32, dev)
    rc = _lib().echo_fp8_quantize(xp, F32 if x.dtype is k.f32[0] else BF16, stride, batch, n, cols,
                                  block_rows, cp, sp, stream_of(stream, dev))
    if rc:
        echo._check(rc, where)


def gemm_workspace_bytes(num_tokens: int, out_features: int, in_features: int) -> int:
    """Enough for every product of up to ``num_tokens`` tokens with such weights."""
    sizes("echo_fp8_gemm_workspace_bytes", num_tokens, out_features, in_features)
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
    where, k = "echo_fp8_gemm", types()
    dev = k.device()
    if x.dim() != 2 or w.dim() != 2:
        refuse(where, f"x has {x.dim()} axes, w {w.dim()}")
    (T, K), N = x.shape, w.shape[0]
    if (T | K | N) >> 31:
        sizes(where, T, K, N)
    kb = -(-K // BLOCK)
    xp = address(where, "x", x, (T, K), k.codes, dev)
    xsp = address(where, "x_scale", x_scale, (T, kb), k.f32, dev)
    wp = address(where, "w", w, (N, K), k.codes, dev)
    wsp = address(where, "w_scale", w_scale, (-(-N // BLOCK), kb), k.f32, dev)
    yp, stride = rows(where, "out", out, (T, N), k.real, dev)
    rp = None
    if residual is not None:
        rp, rs = rows(where, "residual", residual, (T, N), k.real, dev)
        if residual.dtype is not out.dtype or rs != stride:
            refuse(where, "residual has not the type and strides of out")
    sp, sb = scratch(where, workspace, dev)
    rc = _lib().echo_fp8_gemm(xp, xsp, wp, wsp, T, N, K, rp, yp,
                              F32 if out.dtype is k.f32[0] else BF16, stride, sp, sb,
                              stream_of(stream, dev))
    if rc:
        echo._check(rc, where)
