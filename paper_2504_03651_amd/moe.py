"""Python binding of routing and experts (include/echo_moe.h): checks of the
tensors, then the library's calls on PyTorch's current stream."""
from __future__ import annotations

import ctypes

from . import echo, fp8

SYMBOLS = ["echo_moe_route", "echo_moe_experts", "echo_moe_experts_workspace_bytes"]

SCORES = {"softmax": 0, "sigmoid": 1}


class CRouter(ctypes.Structure):
    _fields_ = [(n, ctypes.c_int32) for n in ("num_experts", "top_k", "score", "num_groups",
                                              "top_groups", "group_top", "renormalize")] + [
        ("scale", ctypes.c_float)]


class CExperts(ctypes.Structure):
    _fields_ = [("num_experts", ctypes.c_int32), ("hidden", ctypes.c_int32),
                ("intermediate", ctypes.c_int32),
                ("w_gate_up", ctypes.c_void_p), ("gate_up_scale", ctypes.c_void_p),
                ("w_down", ctypes.c_void_p), ("down_scale", ctypes.c_void_p)]


_bound = False


def _lib():
    global _bound
    L = echo.lib()
    if not _bound:
        vp, i32, i64, sz = ctypes.c_void_p, ctypes.c_int32, ctypes.c_int64, ctypes.c_size_t
        X = ctypes.POINTER(CExperts)
        L.echo_moe_route.argtypes = [ctypes.POINTER(CRouter), vp, i32, i64, i32, vp, vp, vp, vp]
        L.echo_moe_route.restype = ctypes.c_int
        L.echo_moe_experts.argtypes = [X, vp, vp, i32, i32, vp, vp, vp, vp, vp, sz, vp]
        L.echo_moe_experts.restype = ctypes.c_int
        L.echo_moe_experts_workspace_bytes.argtypes = [X, i32, i32]
        L.echo_moe_experts_workspace_bytes.restype = sz
        _bound = True
    return L


class Router:
    """How tokens choose experts (echo_router_t)."""

    def __init__(self, num_experts: int, top_k: int, score: str = "softmax", num_groups: int = 1,
                 top_groups: int = 1, group_top: int = 1, renormalize: bool = False,
                 scale: float = 1.0):
        if score not in SCORES:
            raise echo.EchoError(echo.ECHO_E_UNSUPPORTED, "Router", f"score {score!r}")
        fp8.sizes("Router", num_experts, top_k, num_groups, top_groups, group_top)
        self.num_experts, self.top_k = num_experts, top_k
        self.c = CRouter(num_experts, top_k, SCORES[score], num_groups, top_groups, group_top,
                         int(renormalize), scale)
        self.ref = ctypes.byref(self.c)


def route(router: Router, logits, ids, weights, bias=None, stream=None) -> None:
    """ids (int32) and weights (fp32) [T][top_k] of the experts chosen from
    ``logits`` [T][E] (bf16 or fp32, rows any distance apart); ``bias``: fp32 [E]."""
    where, k = "echo_moe_route", fp8.types()
    dev = k.device()
    if logits.dim() != 2:
        fp8.refuse(where, f"logits has {logits.dim()} axes")
    T, E, n = logits.shape[0], router.num_experts, router.top_k
    if T >> 31:
        fp8.sizes(where, T)
    lp, stride = fp8.rows(where, "logits", logits, (T, E), k.real, dev)
    ip = fp8.address(where, "ids", ids, (T, n), k.i32, dev)
    wp = fp8.address(where, "weights", weights, (T, n), k.f32, dev)
    bp = None if bias is None else fp8.address(where, "bias", bias, (E,), k.f32, dev)
    rc = _lib().echo_moe_route(router.ref, lp, fp8.F32 if logits.dtype is k.f32[0] else fp8.BF16,
                               stride, T, bp, ip, wp, fp8.stream_of(stream, dev))
    if rc:
        echo._check(rc, where)


class Experts:
    """The experts' weights, e4m3 codes and scales: w_gate_up [E][2 I][H] (gate
    rows, then up rows) with scales [E][2][ceil(I/128)][ceil(H/128)], w_down
    [E][H][I] with scales [E][ceil(H/128)][ceil(I/128)]."""

    def __init__(self, w_gate_up, gate_up_scale, w_down, down_scale):
        where, k = "Experts", fp8.types()
        if w_down.dim() != 3:
            fp8.refuse(where, f"w_down has {w_down.dim()} axes")
        E, H, I = w_down.shape
        fp8.sizes(where, E, H, I)
        hb, ib = fp8.blocks(H), fp8.blocks(I)
        self.device = dev = w_down.get_device()
        if dev < 0:
            fp8.refuse(where, "w_down is not on a GPU")
        self.num_experts, self.hidden, self.intermediate = E, H, I
        self.t = (w_gate_up, gate_up_scale, w_down, down_scale)   # kept alive
        self.c = CExperts(E, H, I,
                          fp8.address(where, "w_gate_up", w_gate_up, (E, 2 * I, H), k.codes, dev),
                          fp8.address(where, "gate_up_scale", gate_up_scale, (E, 2, ib, hb), k.f32, dev),
                          fp8.address(where, "w_down", w_down, (E, H, I), k.codes, dev),
                          fp8.address(where, "down_scale", down_scale, (E, hb, ib), k.f32, dev))
        self.ref = ctypes.byref(self.c)

    def workspace_bytes(self, num_tokens: int, top_k: int) -> int:
        fp8.sizes("echo_moe_experts_workspace_bytes", num_tokens, top_k)
        n = int(_lib().echo_moe_experts_workspace_bytes(self.ref, int(num_tokens), int(top_k)))
        if n == 0 and echo.last_error():
            raise echo.EchoError(echo.ECHO_E_INVALID, "echo_moe_experts_workspace_bytes",
                                 echo.last_error())
        return n


def experts(ex: Experts, x, x_scale, ids, weights, out, workspace, residual=None,
            stream=None) -> None:
    """out [T][H] bf16 = (residual +) the weighted sum of the outputs of the
    experts ``ids`` [T][top_k] for x (codes [T][H], scales [T][ceil(H/128)])."""
    where, k = "echo_moe_experts", fp8.types()
    dev = k.device()
    if ex.device != dev:
        fp8.refuse(where, f"the experts are on cuda:{ex.device}, the current device is cuda:{dev}")
    if x.dim() != 2 or ids.dim() != 2:
        fp8.refuse(where, f"x has {x.dim()} axes, ids {ids.dim()}")
    T, H, n = x.shape[0], ex.hidden, ids.shape[1]
    if (T | n) >> 31:
        fp8.sizes(where, T, n)
    xp = fp8.address(where, "x", x, (T, H), k.codes, dev)
    xsp = fp8.address(where, "x_scale", x_scale, (T, -(-H // fp8.BLOCK)), k.f32, dev)
    ip = fp8.address(where, "ids", ids, (T, n), k.i32, dev)
    wp = fp8.address(where, "weights", weights, (T, n), k.f32, dev)
    op = fp8.address(where, "out", out, (T, H), k.bf16, dev)
    rp = None if residual is None else fp8.address(where, "residual", residual, (T, H), k.bf16, dev)
    sp, sb = fp8.scratch(where, workspace, dev)
    rc = _lib().echo_moe_experts(ex.ref, xp, xsp, T, n, ip, wp, rp, op, sp, sb,
                                 fp8.stream_of(stream, dev))
    if rc:
        echo._check(rc, where)
