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
