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
        self.num_experts, self.top_k = num_experts, top_k
        self.c = CRouter(num_experts, top_k, SCORES[score], num_groups, top_groups, group_top,
                         int(renormalize), scale)


def route(router: Router, logits, ids, weights, bias=None, stream=None) -> None:
    """ids (int32) and weights (fp32) [T][top_k] of the experts chosen from
    ``logits`` [T][E] (bf16 or fp32, rows any distance apart); ``bias``: fp32 [E]."""
    where = "echo_moe_route"
    T = logits.shape[0]
    fp8.check(where, "logits", logits, (T, router.num_experts), "real", rows=True)
    fp8.check(where, "ids", ids, (T, router.top_k), "i32")
    fp8.check(where, "weights", weights, (T, router.top_k), "f32")
    if bias is not None:
        fp8.check(where, "bias", bias, (router.num_experts,), "f32")
    echo._check(_lib().echo_moe_route(
        ctypes.byref(router.c), logits.data_ptr(), fp8.real_dtype(logits), fp8.row_stride(logits),
        T, None if bias is None else bias.data_ptr(), ids.data_ptr(), weights.data_ptr(),
        echo._stream(stream)), where)


class Experts:
    """The experts' weights, e4m3 codes and scales: w_gate_up [E][2 I][H] (gate
    rows, then up rows) with scales [E][2][ceil(I/128)][ceil(H/128)], w_down
    [E][H][I] with scales [E][ceil(H/128)][ceil(I/128)]."""

    def __init__(self, w_gate_up, gate_up_scale, w_down, down_scale):
        where = "Experts"
        if w_down.dim() != 3:
            raise echo.EchoError(echo.ECHO_E_INVALID, where, f"w_down has {w_down.dim()} axes")
        E, H, I = w_down.shape
        hb, ib = fp8.blocks(H), fp8.blocks(I)
        fp8.check(where, "w_down", w_down, (E, H, I), "codes")
        fp8.check(where, "w_gate_up", w_gate_up, (E, 2 * I, H), "codes")
        fp8.check(where, "gate_up_scale", gate_up_scale, (E, 2, ib, hb), "f32")
        fp8.check(where, "down_scale", down_scale, (E, hb, ib), "f32")
        self.num_experts, self.hidden, self.intermediate = E, H, I
        self.t = (w_gate_up, gate_up_scale, w_down, down_scale)   # kept alive
        self.c = CExperts(E, H, I, *[x.data_ptr() for x in self.t])

    def workspace_bytes(self, num_tokens: int, top_k: int) -> int:
        n = int(_lib().echo_moe_experts_workspace_bytes(ctypes.byref(self.c), int(num_tokens),
                                                        int(top_k)))
        if n == 0 and echo.last_error():
            raise echo.EchoError(echo.ECHO_E_INVALID, "echo_moe_experts_workspace_bytes",
                                 echo.last_error())
        return n


def experts(ex: Experts, x, x_scale, ids, weights, out, workspace, residual=None,
            stream=None) -> None:
    """out [T][H] bf16 = (residual +) the weighted sum of the outputs of the
    experts ``ids`` [T][top_k] for x (codes [T][H], scales [T][ceil(H/128)])."""
    where = "echo_moe_experts"
    T, H = x.shape
    k = ids.shape[-1]
    fp8.check(where, "x", x, (T, ex.hidden), "codes")
    fp8.check(where, "x_scale", x_scale, (T, fp8.blocks(H)), "f32")
    fp8.check(where, "ids", ids, (T, k), "i32")
    fp8.check(where, "weights", weights, (T, k), "f32")
    fp8.check(where, "out", out, (T, H), "bf16")
    fp8.on_device(where, "w_down", ex.t[2])
    if residual is not None:
        fp8.check(where, "residual", residual, (T, H), "bf16")
    wp, wb = fp8._workspace(where, workspace)
    echo._check(_lib().echo_moe_experts(
        ctypes.byref(ex.c), x.data_ptr(), x_scale.data_ptr(), T, k, ids.data_ptr(),
        weights.data_ptr(), None if residual is None else residual.data_ptr(), out.data_ptr(),
        wp, wb, echo._stream(stream)), where)
