"""The layer with experts refuses before anything is enqueued (CPU)."""
import ctypes

import pytest

from paper_2504_03651_amd import echo, moe, workload as W
from tests.test_fp8_host import CALL, EXPERTS, INV, P, _moe_layer, at


@pytest.mark.parametrize("scale", ["gate_up_scale", "down_scale"])
def test_expert_scales_off_their_alignment(scale):
    """Seen by the experts' check of no tokens, which the layer makes first."""
    ex = moe.CExperts(*{**EXPERTS, scale: at(2)}.values())
    none = {**CALL, "T": 0}
    rc = moe._lib().echo_moe_experts(ctypes.byref(ex), *none.values(), None, 0, None)
    assert rc == INV and "aligned" in echo.last_error()
    layer, c = _moe_layer(experts=ex)
    cp, cb, keep = echo.host_structs(W.config1())
    args = (ctypes.byref(c), ctypes.byref(cp), ctypes.byref(cb))
    assert layer._lib().echo_moe_layer_workspace_bytes(*args) == 0 and "aligned" in echo.last_error()
    assert layer._lib().echo_moe_layer_forward(*args, P, P, 1 << 40, None, 0, None) == INV
    assert "aligned" in echo.last_error()


def _dense():
    from paper_2504_03651_amd import layer
    return layer, layer.CLayer(256, 4, 4, 64, 128, 1e4, 1e-5, P, P, P, P, P, P)


@pytest.mark.parametrize("name", ["echo_moe_layer_forward", "echo_layer_forward"])
@pytest.mark.parametrize("short", [None, 16])
def test_host_workspace_is_checked_before_anything_is_enqueued(name, short):
    """The attention's plan needs host memory: a layer without it, or with too little,
    is refused before the cache is touched (before any library handle or launch, too:
    there is no GPU here)."""
    layer, c = _moe_layer() if "moe" in name else _dense()
    cp, cb, keep = echo.host_structs(W.config1())
    need = echo.lib().echo_attn_host_workspace_bytes(ctypes.byref(cp), ctypes.byref(cb), 4)
    assert need > 16
    host = ctypes.create_string_buffer(64)
    rc = getattr(layer._lib(), name)(ctypes.byref(c), ctypes.byref(cp), ctypes.byref(cb), P, P, 1 << 40,
                                     None if short is None else ctypes.addressof(host), short or 0, None)
    assert rc == echo.ECHO_E_WORKSPACE and "host workspace" in echo.last_error(), echo.last_error()


@pytest.mark.parametrize("name, tokens, inter", [("moe", 1 << 24, 144), ("dense", 1 << 24, 128), ("dense", 1 << 21, 1 << 14)])
def test_more_tokens_than_a_launch_holds(name, tokens, inter):
    """2^32 threads, at 256 a token, or at one for eight activations of the MLP."""
    layer, c = _moe_layer() if name == "moe" else _dense()
    if name == "dense":
        c.intermediate = inter
    cp, cb, keep = echo.host_structs(W.config1())
    for f in ("h_block_tables", "h_seq_lens", "h_q_start", "h_row_kind"):
        setattr(cb, f, None)
    ask = getattr(layer._lib(), f"echo_{'moe_' if name == 'moe' else ''}layer_workspace_bytes")
    args = (ctypes.byref(c), ctypes.byref(cp), ctypes.byref(cb))
    assert ask(*args) > 0
    cb.num_tokens = tokens
    assert ask(*args) == 0 and "more than a launch holds" in echo.last_error()
