"""Host-side checks of the 8-bit products, the router and the experts (CPU): the
library exports what the headers declare, refuses what they forbid before any
GPU work, and sizes workspaces; and the reference's own codec and rules."""
import ctypes
import os
import re

import numpy as np
import pytest

from oracle import fp8_oracle as FO
from paper_2504_03651_amd import echo, fp8, moe
from tests.bruteforce import e4m3_table

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
P = ctypes.c_void_p(1 << 20)   # an aligned stand-in for device memory, never touched
INV, UNS, WSP = echo.ECHO_E_INVALID, echo.ECHO_E_UNSUPPORTED, echo.ECHO_E_WORKSPACE


def at(offset):
    return ctypes.c_void_p((1 << 20) + offset)


@pytest.mark.parametrize("header, mod", [("echo_fp8.h", fp8), ("echo_moe.h", moe)])
def test_library_exports_every_declared_symbol(header, mod):
    text = open(os.path.join(ROOT, "include", header)).read()
    text = re.sub(r"/\*.*?\*/", "", text, flags=re.S)
    declared = set(re.findall(r"\b(echo_[a-z0-9_]+)\s*\(", text))
    assert declared == set(mod.SYMBOLS)
    for name in declared:
        assert hasattr(echo.lib(), name), name


def test_reference_codec():
    assert np.array_equal(FO.TABLE, e4m3_table(), equal_nan=True)
    c = np.array([i for i in range(256) if i not in (0x7F, 0xFF)])
    assert np.array_equal(FO.encode(FO.TABLE[c]), c)
    assert list(FO.encode([17.0, 19.0, 464.0, 1e9, -1e9, np.nan, 2.0 ** -10])) == \
        [0x58, 0x5A, 0x7E, 0x7E, 0xFE, 0x7F, 0x00]   # ties to even, saturation


def test_reference_router_on_a_row_by_hand():
    z = np.log(np.array([[0.1, 0.2, 0.3, 0.4]]))
    i, w = FO.route(z, 2)
    assert i.tolist() == [[3, 2]] and np.allclose(w, [[0.4, 0.3]])
    i, w = FO.route(z, 2, bias=np.array([0.0, 0.25, 0.0, 0.0]), renormalize=True, scale=2.0)
    assert i.tolist() == [[1, 3]] and np.allclose(w, [[2 / 3, 4 / 3]])
    i, w = FO.route(z, 2, num_groups=2, top_groups=1, bias=np.array([1.0, 0, 0, 0]))
    assert i.tolist() == [[0, 1]]
    i, w = FO.route(np.array([[1.0, np.nan, -np.inf, 1.0]]), 3)
    assert i.tolist() == [[0, 3, -1]] and np.allclose(w, [[0.5, 0.5, 0.0]])


QUANT = dict(x=P, x_dtype=0, x_stride=256, batch=1, rows=4, cols=256, block_rows=1, codes=P, scales=P)


@pytest.mark.parametrize("change, code, what", [
    (dict(x=None), INV, "NULL"), (dict(codes=None), INV, "NULL"), (dict(scales=None), INV, "NULL"),
    (dict(x_dtype=2), UNS, "dtype"), (dict(rows=-1), INV, "rows"), (dict(batch=-1), INV, "batch"),
    (dict(cols=0), INV, "cols"), (dict(cols=250), UNS, "multiple of 16"),
    (dict(block_rows=64), UNS, "block_rows"), (dict(x_stride=255), INV, "x_stride"),
    (dict(x_stride=260), INV, "x_stride"), (dict(x_dtype=1, x_stride=258), INV, "x_stride"),
    (dict(x=at(8)), INV, "aligned"), (dict(codes=at(8)), INV, "aligned"),
    (dict(scales=at(2)), INV, "aligned"),
    (dict(batch=2 ** 20, rows=2 ** 20), UNS, "blocks"),
])
def test_quantize_refusals(change, code, what):
    rc = fp8._lib().echo_fp8_quantize(*{**QUANT, **change}.values(), None)
    assert rc == code and what in echo.last_error(), echo.last_error()


GEMM = dict(x=P, xs=P, w=P, ws=P, T=4, N=100, K=256, res=None, y=P, dtype=0, stride=100)


@pytest.mark.parametrize("change, code, what", [
    (dict(x=None), INV, "NULL"), (dict(xs=None), INV, "NULL"), (dict(w=None), INV, "NULL"),
    (dict(ws=None), INV, "NULL"), (dict(y=None), INV, "NULL"), (dict(T=-1), INV, "num_tokens"),
    (dict(N=0), INV, "out_features"), (dict(K=0), INV, "in_features"),
    (dict(K=250), UNS, "multiple of 16"), (dict(dtype=2), UNS, "dtype"),
    (dict(stride=99), INV, "y_stride"), (dict(x=at(8)), INV, "16-byte"),
    (dict(w=at(4)), INV, "16-byte"), (dict(xs=at(2)), INV, "alignment"),
    (dict(y=at(1)), INV, "alignment"), (dict(dtype=1, res=at(2)), INV, "alignment"),
    (dict(T=2 ** 31 - 1, N=2 ** 31 - 1, stride=2 ** 31), UNS, "too large"),
    (dict(T=1, N=2 ** 30 + 1, stride=2 ** 31), UNS, "too large"), (dict(K=2 ** 23 + 16), UNS, "above"),
])
def test_gemm_refusals(change, code, what):
    rc = fp8._lib().echo_fp8_gemm(*{**GEMM, **change}.values(), P, 1 << 40, None)
    assert rc == code and what in echo.last_error(), echo.last_error()


def test_gemm_workspace():
    L = fp8._lib()
    for T, N, K in [(1, 16, 16), (137, 4096, 14336), (4640, 28672, 4096)]:
        n = fp8.gemm_workspace_bytes(T, N, K)
        if n:
            for ws, nb in [(None, n), (P, n - 1), (at(128), n)]:
                rc = L.echo_fp8_gemm(*{**GEMM, "T": T, "N": N, "K": K, "stride": N}.values(), ws, nb, None)
                assert rc == WSP, echo.last_error()
    with pytest.raises(echo.EchoError):
        fp8.gemm_workspace_bytes(1, 16, 17)


ROUTER = dict(num_experts=64, top_k=8, score=0, num_groups=8, top_groups=4, group_top=2,
              renormalize=1, scale=1.0)
ROUTE = dict(logits=P, dtype=0, stride=64, T=4, bias=P, ids=P, weights=P)


@pytest.mark.parametrize("router, call, code, what", [
    (dict(num_experts=0), {}, UNS, "num_experts"), (dict(num_experts=520), {}, UNS, "num_experts"),
    (dict(score=2), {}, UNS, "score"), (dict(num_groups=0), {}, INV, "num_groups"),
    (dict(num_groups=7), {}, INV, "num_groups"), (dict(num_experts=512, num_groups=128), {}, INV, "num_groups"),
    (dict(top_groups=0), {}, INV, "top_groups"), (dict(top_groups=9), {}, INV, "top_groups"),
    (dict(group_top=0), {}, INV, "group_top"), (dict(group_top=3), {}, INV, "group_top"),
    (dict(num_groups=64, top_groups=64), {}, INV, "group_top"),
    (dict(top_k=0), {}, INV, "top_k"), (dict(top_groups=1, top_k=9), {}, INV, "top_k"),
    (dict(num_experts=512, top_groups=8, top_k=65), dict(stride=512), INV, "top_k"),
    (dict(scale=float("nan")), {}, INV, "scale"), (dict(scale=float("inf")), {}, INV, "scale"),
    ({}, dict(logits=None), INV, "NULL"), ({}, dict(ids=None), INV, "NULL"),
    ({}, dict(weights=None), INV, "NULL"), ({}, dict(dtype=3), UNS, "dtype"),
    ({}, dict(stride=63), INV, "logits_stride"), ({}, dict(T=-1), INV, "num_tokens"),
    ({}, dict(logits=at(1)), INV, "aligned"), ({}, dict(dtype=1, logits=at(2)), INV, "aligned"),
    ({}, dict(bias=at(2)), INV, "aligned"), ({}, dict(ids=at(1)), INV, "aligned"),
])
def test_route_refusals(router, call, code, what):
    c = moe.CRouter(*{**ROUTER, **router}.values())
    rc = moe._lib().echo_moe_route(ctypes.byref(c), *{**ROUTE, **call}.values(), None)
    assert rc == code and what in echo.last_error(), echo.last_error()
    assert moe._lib().echo_moe_route(None, *ROUTE.values(), None) == INV


EXPERTS = dict(num_experts=8, hidden=256, intermediate=144, w_gate_up=P, gate_up_scale=P, w_down=P,
               down_scale=P)
CALL = dict(x=P, xs=P, T=5, top_k=2, ids=P, weights=P, residual=None, out=P)


@pytest.mark.parametrize("ex, call, code, what", [
    (dict(num_experts=0), {}, UNS, "num_experts"), (dict(num_experts=513), {}, UNS, "num_experts"),
    (dict(hidden=0), {}, INV, "hidden"), (dict(intermediate=-16), {}, INV, "intermediate"),
    (dict(hidden=250), {}, UNS, "multiples of 16"), (dict(intermediate=100), {}, UNS, "multiples of 16"),
    (dict(w_gate_up=None), {}, INV, "NULL"), (dict(gate_up_scale=None), {}, INV, "NULL"),
    (dict(w_down=None), {}, INV, "NULL"), (dict(down_scale=None), {}, INV, "NULL"),
    (dict(w_gate_up=at(8)), {}, INV, "16-byte"), (dict(w_down=at(8)), {}, INV, "16-byte"),
    (dict(down_scale=at(2)), {}, INV, "aligned"),
    ({}, dict(T=-1), INV, "num_tokens"), ({}, dict(top_k=0), INV, "top_k"),
    ({}, dict(top_k=65), INV, "top_k"), ({}, dict(T=1 << 24), UNS, "pairs"),
    (dict(hidden=1 << 16, intermediate=1 << 15), {}, UNS, "2^32"), (dict(hidden=1 << 12), dict(T=1 << 20), UNS, "2^32"),
    ({}, dict(x=None), INV, "NULL"), ({}, dict(xs=None), INV, "NULL"), ({}, dict(ids=None), INV, "NULL"),
    ({}, dict(weights=None), INV, "NULL"), ({}, dict(out=None), INV, "NULL"),
    ({}, dict(x=at(8)), INV, "16-byte"), ({}, dict(out=at(2)), INV, "16-byte"),
    ({}, dict(residual=at(8)), INV, "16-byte"), ({}, dict(ids=at(2)), INV, "aligned"),
])
def test_experts_refusals(ex, call, code, what):
    c = moe.CExperts(*{**EXPERTS, **ex}.values())
    rc = moe._lib().echo_moe_experts(ctypes.byref(c), *{**CALL, **call}.values(), P, 1 << 40, None)
    assert rc == code and what in echo.last_error(), echo.last_error()


def test_experts_workspace():
    c = moe.CExperts(*EXPERTS.values())
    L = moe._lib()
    n = L.echo_moe_experts_workspace_bytes(ctypes.byref(c), 5, 2)
    assert n > 0
    for ws, nb in [(None, n), (P, n - 1), (at(128), n)]:
        assert L.echo_moe_experts(ctypes.byref(c), *CALL.values(), ws, nb, None) == WSP
    assert L.echo_moe_experts_workspace_bytes(ctypes.byref(c), 0, 2) == 0 and not echo.last_error()
    assert L.echo_moe_experts_workspace_bytes(None, 5, 2) == 0 and echo.last_error()
    # no tokens: nothing to do, no buffers needed
    none = {**CALL, "T": 0, "x": None, "xs": None, "ids": None, "weights": None, "out": None}
    assert L.echo_moe_experts(ctypes.byref(c), *none.values(), None, 0, None) == 0
    r = moe.CRouter(*ROUTER.values())
    assert L.echo_moe_route(ctypes.byref(r), None, 0, 64, 0, None, None, None, None) == 0
    assert fp8._lib().echo_fp8_quantize(None, 0, 256, 1, 0, 256, 1, None, None, None) == 0
    assert fp8._lib().echo_fp8_gemm(*{**GEMM, "T": 0, "x": None, "y": None}.values(), None, 0, None) == 0


def test_binding_refuses_host_tensors_and_wrong_layouts():
    import torch
    x = torch.zeros(4, 256, dtype=torch.bfloat16)
    codes, scales = torch.zeros(4, 256, dtype=torch.uint8), torch.zeros(4, 2)
    with pytest.raises(echo.EchoError, match="not on a GPU"):
        fp8.quantize(x, codes, scales)
    with pytest.raises(echo.EchoError, match="block_rows"):
        fp8.quantize(x, codes, scales, block_rows=2)
    with pytest.raises(echo.EchoError, match="dtype"):
        fp8.quantize(x.half(), codes, scales)
    with pytest.raises(echo.EchoError, match="shape"):
        moe.route(moe.Router(64, 4), x, scales, scales)
    with pytest.raises(echo.EchoError, match="score"):
        moe.Router(64, 4, score="tanh")


def _moe_layer(**change):
    from paper_2504_03651_amd import layer
    v = dict(hidden=256, num_q_heads=4, num_kv_heads=4, head_dim=64, rope_theta=1e4, rms_eps=1e-5,
             attn_norm=P, w_qkv=P, w_o=P, mlp_norm=P, w_router=P, w_qkv_scale=P, w_o_scale=P,
             router_bias=None, router=moe.CRouter(8, 2, 0, 1, 1, 1, 0, 1.0),
             experts=moe.CExperts(*EXPERTS.values()))
    return layer, layer.CMoELayer(*{**v, **change}.values())


@pytest.mark.parametrize("change, code, what", [
    (dict(hidden=0), INV, "shape"), (dict(hidden=264), UNS, "multiple of 16"),
    (dict(num_q_heads=6), INV, "shape"), (dict(head_dim=128), INV, "differ from the pool"),
    (dict(w_qkv=None), INV, "NULL"), (dict(w_o_scale=None), INV, "NULL"), (dict(w_router=None), INV, "NULL"),
    (dict(router=moe.CRouter(4, 2, 0, 1, 1, 1, 0, 1.0)), INV, "experts"),
    (dict(router=moe.CRouter(8, 9, 0, 1, 1, 1, 0, 1.0)), INV, "top_k"),
    (dict(hidden=272), INV, "experts"),
    (dict(experts=moe.CExperts(*{**EXPERTS, "w_down": None}.values())), INV, "NULL"),
    (dict(attn_norm=at(8)), INV, "16-byte"), (dict(w_o_scale=at(2)), INV, "4-byte"),
])
def test_moe_layer_refusals(change, code, what):
    from paper_2504_03651_amd import workload as W
    layer, c = _moe_layer(**change)
    cp, cb, keep = echo.host_structs(W.config1())
    rc = layer._lib().echo_moe_layer_forward(ctypes.byref(c), ctypes.byref(cp), ctypes.byref(cb), P, P, 1 << 40,
                                             None, 0, None)
    assert rc == code and what in echo.last_error(), echo.last_error()


def test_moe_layer_workspace():
    from paper_2504_03651_amd import workload as W
    layer, c = _moe_layer()
    cp, cb, keep = echo.host_structs(W.config1())
    args = (ctypes.byref(c), ctypes.byref(cp), ctypes.byref(cb))
    n = layer._lib().echo_moe_layer_workspace_bytes(*args)
    assert n > 0
    for hidden, ws, nb, code in [(None, P, n, INV), (P, None, n, WSP), (P, P, n - 1, WSP), (P, at(128), n, WSP)]:
        assert layer._lib().echo_moe_layer_forward(*args, hidden, ws, nb, None, 0, None) == code
    cb.num_tokens += 1
    assert layer._lib().echo_moe_layer_workspace_bytes(*args) == 0 and echo.last_error()
