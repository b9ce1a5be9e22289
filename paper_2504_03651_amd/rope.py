"""Python binding of the rotary positions (include/echo_rope.h): checks of the tensors,
then the library's calls on PyTorch's current stream."""
from __future__ import annotations

import ctypes

from . import echo, fp8
from .fp8 import BF16, F32, address, refuse, sizes, stream_of

SYMBOLS = ["echo_rope_frequencies", "echo_rope_rotate"]

LAYOUTS = {"half": 0, "interleaved": 1}
SCALINGS = {"none": 0, "linear": 1, "ntk": 2, "bands": 3, "yarn": 4}


class CRope(ctypes.Structure):
    _fields_ = [*[(n, ctypes.c_int32) for n in ("head_dim", "rotary_dim", "layout", "scaling")],
                *[(n, ctypes.c_double) for n in ("theta", "factor", "low", "high")],
                ("original_length", ctypes.c_int32)]


class CHeads(ctypes.Structure):
    _fields_ = [("in_", ctypes.c_void_p), ("out", ctypes.c_void_p), ("heads", ctypes.c_int32),
                *[(n, ctypes.c_int64) for n in ("in_token", "in_head", "out_token", "out_head")]]


_bound = False


def _lib():
    global _bound
    L = echo.lib()
    if not _bound:
        vp, i32, f64 = ctypes.c_void_p, ctypes.c_int32, ctypes.c_double
        R, D = ctypes.POINTER(CRope), ctypes.POINTER(ctypes.c_double)
        L.echo_rope_frequencies.argtypes = [R, D, D]
        L.echo_rope_frequencies.restype = ctypes.c_int
        L.echo_rope_rotate.argtypes = [R, vp, f64, vp, i32, i32, ctypes.POINTER(CHeads), i32, i32, vp]
        L.echo_rope_rotate.restype = ctypes.c_int
        _bound = True
    return L


class Rope:
    """How heads are turned (echo_rope_t), with its frequencies on ``device``.

    ``scaling``: "none", "linear", "ntk", "bands" or "yarn" by ``factor``, the last two
    with the turns ``low`` and ``high`` over ``original_length``.  ``frequencies`` (radians
    a position, [rotary_dim / 2]) and ``magnitude`` take the place of the computed ones."""

    def __init__(self, head_dim: int, rotary_dim: int | None = None, layout: str = "half",
                 theta: float = 10000.0, scaling: str = "none", factor: float = 1.0,
                 low: float = 1.0, high: float = 32.0, original_length: int = 0,
                 frequencies=None, magnitude: float | None = None, device="cuda"):
        import torch
        where = "Rope"
        for name, value, known in (("layout", layout, LAYOUTS), ("scaling", scaling, SCALINGS)):
            if value not in known:
                raise echo.EchoError(echo.ECHO_E_UNSUPPORTED, where, f"{name} {value!r}")
        rotary_dim = head_dim if rotary_dim is None else rotary_dim
        sizes(where, head_dim, rotary_dim, original_length)
        self.head_dim, self.rotary_dim = head_dim, rotary_dim
        self.c = CRope(head_dim, rotary_dim, LAYOUTS[layout], SCALINGS[scaling], theta, factor, low, high,
                       original_length)
        self.ref = ctypes.byref(self.c)
        f, m = (ctypes.c_double * max(1, rotary_dim // 2))(), ctypes.c_double()
        echo._check(_lib().echo_rope_frequencies(self.ref, f, ctypes.byref(m)), "echo_rope_frequencies")
        if frequencies is None:
            frequencies = list(f)
        self.frequencies = torch.as_tensor(frequencies, dtype=torch.float64, device=device).contiguous()
        if self.frequencies.shape != (rotary_dim // 2,):
            refuse(where, f"frequencies has shape {tuple(self.frequencies.shape)}, not {(rotary_dim // 2,)}")
        self.magnitude = float(m.value if magnitude is None else magnitude)


def _heads(where, name, x, T, D, dtypes, dev):
    """(address, heads, elements from token to token and from head to head)"""
    if x.dim() != 3 or x.shape[0] != T or x.shape[2] != D:
        refuse(where, f"{name} has shape {tuple(x.shape)}, not ({T}, heads, {D})")
    if x.dtype not in dtypes:
        refuse(where, f"{name} has dtype {x.dtype}")
    if x.get_device() != dev:
        fp8._place(where, name, x, dev)
    t, h, one = x.stride()
    if one != 1:
        refuse(where, f"the columns of {name} are not adjacent")
    n = x.shape[1]
    if n >> 31:
        sizes(where, n)
    # an axis of one has any stride
    return x.data_ptr(), n, t if T > 1 else n * D, h if n > 1 else D


def rotate(rope: Rope, positions, q, k=None, q_out=None, k_out=None, inverse: bool = False,
           stream=None) -> None:
    """Turns the heads of q [T][heads][D] and of k (bf16 or fp32, both alike, tokens and
    heads any distance apart) by ``positions`` (int32 [T]), into q_out and k_out or in
    place."""
    where, ty = "echo_rope_rotate", fp8.types()
    dev = ty.device()
    if q.dim() != 3:
        refuse(where, f"q has {q.dim()} axes")
    T, D = q.shape[0], rope.head_dim
    if T >> 31:
        sizes(where, T)
    if q.dtype not in ty.real:
        refuse(where, f"q has dtype {q.dtype}")
    dtypes = (q.dtype,)
    if k is None and k_out is not None:
        refuse(where, "k_out without k")
    tensors = (CHeads * 2)()
    n = 0
    for name, x, out in (("q", q, q_out), ("k", k, k_out)):
        if x is None:
            continue
        xp, heads, xt, xh = _heads(where, name, x, T, D, dtypes, dev)
        op, ot, oh = xp, xt, xh
        if out is not None:
            op, out_heads, ot, oh = _heads(where, name + "_out", out, T, D, dtypes, dev)
            if out_heads != heads:
                refuse(where, f"{name}_out has {out_heads} heads, {name} {heads}")
        tensors[n] = CHeads(xp, op, heads, xt, xh, ot, oh)
        n += 1
    pp = address(where, "positions", positions, (T,), ty.i32, dev)
    f = rope.frequencies
    if f.get_device() != dev:
        fp8._place(where, "rope.frequencies", f, dev)
    rc = _lib().echo_rope_rotate(rope.ref, f.data_ptr(), rope.magnitude, pp, T,
                                 F32 if q.dtype is ty.f32[0] else BF16, tensors, n, int(inverse),
                                 stream_of(stream, dev))
    if rc:
        echo._check(rc, where)
