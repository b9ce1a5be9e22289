"""Python binding of the rotary positions (include/echo_rope.h): checks of the tensors,
then the library's calls on PyTorch's current stream."""
from __future__ import annotations

import ctypes

from . import echo, native
from .fp8 import refuse, sizes

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
        self.at = ctypes.addressof(self.c)
        f, m = (ctypes.c_double * max(1, rotary_dim // 2))(), ctypes.c_double()
        echo._check(_lib().echo_rope_frequencies(ctypes.byref(self.c), f, ctypes.byref(m)), "echo_rope_frequencies")
        if frequencies is None:
            frequencies = list(f)
        self.frequencies = torch.as_tensor(frequencies, dtype=torch.float64, device=device).contiguous()
        if self.frequencies.shape != (rotary_dim // 2,):
            refuse(where, f"frequencies has shape {tuple(self.frequencies.shape)}, not {(rotary_dim // 2,)}")
        self.magnitude = float(m.value if magnitude is None else magnitude)

    def __setstate__(self, state):
        """Of a copy, in this process or another: its description has an address of its own."""
        self.__dict__.update(state)
        self.at = ctypes.addressof(self.c)


def rotate(rope: Rope, positions, q, k=None, q_out=None, k_out=None, inverse: bool = False,
           stream=None) -> None:
    """Turns the heads of q [T][heads][D] and of k (bf16 or fp32, both alike, tokens and
    heads any distance apart) by ``positions`` (int32 [T]), into q_out and k_out or in
    place."""
    native.binding().rotate(rope.at, rope.frequencies, rope.magnitude, positions, q, k, q_out, k_out, inverse,
                            stream)
