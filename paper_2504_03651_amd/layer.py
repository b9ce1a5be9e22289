"""Python binding of the decoder layers (include/echo_layer.h): marshalling only.

Uploads a layer's weights to device memory with PyTorch (``MoELayer`` quantises
them there) and calls echo_layer_forward or echo_moe_layer_forward on PyTorch's
current stream; every step runs in the library (HIP kernels and hipBLASLt).
"""
from __future__ import annotations

import ctypes

import numpy as np

from . import echo, fp8, moe

SYMBOLS = ["echo_layer_workspace_bytes", "echo_layer_forward", "echo_layer_timing",
           "echo_moe_layer_workspace_bytes", "echo_moe_layer_forward"]


class CLayer(ctypes.Structure):
    _fields_ = [("hidden", ctypes.c_int32), ("num_q_heads", ctypes.c_int32),
                ("num_kv_heads", ctypes.c_int32), ("head_dim", ctypes.c_int32),
                ("intermediate", ctypes.c_int32), ("rope_theta", ctypes.c_float),
                ("rms_eps", ctypes.c_float),
                ("attn_norm", ctypes.c_void_p), ("w_qkv", ctypes.c_void_p),
                ("w_o", ctypes.c_void_p), ("mlp_norm", ctypes.c_void_p),
                ("w_gate_up", ctypes.c_void_p), ("w_down", ctypes.c_void_p)]


class CMoELayer(ctypes.Structure):
    _fields_ = [("hidden", ctypes.c_int32), ("num_q_heads", ctypes.c_int32),
                ("num_kv_heads", ctypes.c_int32), ("head_dim", ctypes.c_int32),
                ("rope_theta", ctypes.c_float), ("rms_eps", ctypes.c_float),
                *[(n, ctypes.c_void_p) for n in ("attn_norm", "w_qkv", "w_o", "mlp_norm", "w_router",
                                                 "w_qkv_scale", "w_o_scale", "router_bias")],
                ("router", moe.CRouter), ("experts", moe.CExperts)]


class CLayerTiming(ctypes.Structure):
    _fields_ = [(n, ctypes.c_float) for n in ("norm_ms", "qkv_ms", "rope_ms", "append_ms",
                                              "attention_ms", "o_ms", "mlp_ms", "other_ms")]


_bound = False


def _lib():
    global _bound
    L = echo.lib()
    if not _bound:
        P, B, vp = ctypes.POINTER(CLayer), ctypes.POINTER(echo.CPool), ctypes.c_void_p
        L.echo_layer_workspace_bytes.argtypes = [P, B, ctypes.POINTER(echo.CBatch)]
        L.echo_layer_workspace_bytes.restype = ctypes.c_size_t
        L.echo_layer_forward.argtypes = [P, B, ctypes.POINTER(echo.CBatch), vp, vp,
                                         ctypes.c_size_t, vp, ctypes.c_size_t, vp]
        L.echo_layer_forward.restype = ctypes.c_int
        Q = ctypes.POINTER(CMoELayer)
        L.echo_moe_layer_workspace_bytes.argtypes = [Q, B, ctypes.POINTER(echo.CBatch)]
        L.echo_moe_layer_workspace_bytes.restype = ctypes.c_size_t
        L.echo_moe_layer_forward.argtypes = [Q, *L.echo_layer_forward.argtypes[1:]]
        L.echo_moe_layer_forward.restype = ctypes.c_int
        L.echo_layer_timing.argtypes = [ctypes.POINTER(CLayerTiming)]
        L.echo_layer_timing.restype = ctypes.c_int
        _bound = True
    return L


class Layer:
    """Device copy of a ``workload.LayerWeights``."""

    def __init__(self, lw, device: str = "cuda"):
        import torch
        self.lw = lw
        dev = lambda a: torch.from_numpy(np.ascontiguousarray(a).view(np.int16)).to(device)
        self.t = {n: dev(getattr(lw, n)) for n in ("attn_norm", "w_qkv", "w_o", "mlp_norm",
                                                    "w_gate_up", "w_down")}
        self.c = CLayer(lw.hidden, lw.num_q_heads, lw.num_kv_heads, lw.head_dim, lw.intermediate,
                        lw.rope_theta, lw.rms_eps,
                        *[self.t[n].data_ptr() for n in ("attn_norm", "w_qkv", "w_o", "mlp_norm",
                                                         "w_gate_up", "w_down")])

    def workspace_bytes(self, pool, batch) -> int:
        return _workspace_bytes("echo_layer_workspace_bytes", self.c, pool, batch)

    def forward(self, pool, batch, hidden, workspace, stream=None, host_workspace=None) -> None:
        """hidden: device int16 tensor [T][H] (bf16 bits), overwritten.  The
        attention plan goes through ``host_workspace`` (the calling thread's
        pinned ring by default) when the batch has host mirrors."""
        _forward("echo_layer_forward", self.c, self.lw.num_q_heads, pool, batch, hidden, workspace,
                 stream, host_workspace)


def _workspace_bytes(name, c, pool, batch) -> int:
    cp, cb = pool.c(), batch.c()
    n = getattr(_lib(), name)(ctypes.byref(c), ctypes.byref(cp), ctypes.byref(cb))
    if n == 0:
        raise echo.EchoError(echo.ECHO_E_INVALID, name, echo.last_error())
    return int(n)


def _forward(name, c, num_q_heads, pool, batch, hidden, workspace, stream, host_workspace) -> None:
    import torch
    cp, cb = pool.c(), batch.c()
    s = torch.cuda.current_stream() if stream is None else stream
    hptr, hsize, slot, hw = None, 0, None, None
    if batch.mirrors and batch.num_rows:
        hw = host_workspace or echo.default_host_workspace()
        hptr, hsize, slot = hw.acquire(echo.host_workspace_bytes(pool, batch, num_q_heads))
    echo._check(getattr(_lib(), name)(
        ctypes.byref(c), ctypes.byref(cp), ctypes.byref(cb), hidden.data_ptr(),
        workspace.data_ptr(), workspace.numel() * workspace.element_size(),
        hptr, hsize, ctypes.c_void_p(s.cuda_stream)), name)
    if slot is not None:
        hw.release(slot, s)


class MoELayer:
    """Device copy of a ``workload.MoELayerWeights``, its projections and experts
    quantised to e4m3 there, with the router that chooses the experts."""

    def __init__(self, lw, router, device: str = "cuda"):
        import torch
        self.lw, self.router = lw, router
        dev = lambda a: torch.from_numpy(np.ascontiguousarray(a).view(np.int16)).to(device)
        bits = lambda a: dev(a).view(torch.bfloat16)

        def quantized(a, batch=None):
            """Codes and scales of [N][K], or of ``batch`` stacked matrices."""
            x = bits(a) if batch is None else bits(a).reshape(batch, -1, a.shape[-1])
            codes = torch.empty(x.shape, dtype=torch.float8_e4m3fn, device=device)
            scales = torch.empty((*x.shape[:-2], *map(fp8.blocks, x.shape[-2:])), device=device)
            fp8.quantize(x, codes, scales, fp8.BLOCK)
            return codes, scales

        E, H, I = lw.num_experts, lw.hidden, lw.intermediate
        gu, gus = quantized(lw.w_gate_up, 2 * E)
        down, downs = quantized(lw.w_down, E)
        self.experts = moe.Experts(gu.reshape(E, 2 * I, H), gus.reshape(E, 2, *gus.shape[1:]), down, downs)
        self.t = {n: dev(getattr(lw, n)) for n in ("attn_norm", "mlp_norm", "w_router")}
        for n in ("w_qkv", "w_o"):
            self.t[n], self.t[n + "_scale"] = quantized(getattr(lw, n))
        self.t["router_bias"] = torch.from_numpy(np.ascontiguousarray(lw.router_bias, np.float32)).to(device)
        self.c = CMoELayer(H, lw.num_q_heads, lw.num_kv_heads, lw.head_dim, lw.rope_theta, lw.rms_eps,
                           *[self.t[n].data_ptr() for n, _ in CMoELayer._fields_[6:14]],
                           router.c, self.experts.c)

    def workspace_bytes(self, pool, batch) -> int:
        return _workspace_bytes("echo_moe_layer_workspace_bytes", self.c, pool, batch)

    def forward(self, pool, batch, hidden, workspace, stream=None, host_workspace=None) -> None:
        """As ``Layer.forward``."""
        _forward("echo_moe_layer_forward", self.c, self.lw.num_q_heads, pool, batch, hidden, workspace,
                 stream, host_workspace)


def timing() -> dict:
    t = CLayerTiming()
    echo._check(_lib().echo_layer_timing(ctypes.byref(t)), "echo_layer_timing")
    return {n: float(getattr(t, n)) for n, _ in CLayerTiming._fields_}
