"""Sizes of the experts' workspace, and sizes that the kernels cannot address (CPU)."""
import ctypes

import numpy as np
import pytest

from paper_2504_03651_amd import moe
from tests.test_fp8_host import EXPERTS


@pytest.mark.parametrize("E, H, I", [(512, 16, 16), (512, 2048, 512), (64, 2048, 1024), (8, 4096, 14336), (1, 16, 16)])
@pytest.mark.parametrize("top_k", [1, 8])
def test_experts_workspace_does_not_fall_with_the_tokens(E, H, I, top_k):
    """Across the changes of the tiles' size, at 4, 12 and 72 pairs an expert."""
    c = moe.CExperts(*{**EXPERTS, "num_experts": E, "hidden": H, "intermediate": I}.values())
    ask = moe._lib().echo_moe_experts_workspace_bytes
    need = [ask(ctypes.byref(c), t, top_k) for t in range(0, 100 * E // top_k + 40)]
    assert (np.diff(need) >= 0).all(), int(np.argmin(np.diff(need)))


@pytest.mark.parametrize("E, H, I, T, top_k", [(1, 16, 1 << 26, 97, 1), (1, 16, 1 << 26, 13, 1), (8, 16, (1 << 23) + 16, 1, 2)])
def test_experts_refuse_rows_past_32_bit_offsets(E, H, I, T, top_k):
    """Offsets inside a tile of activation rows of `intermediate` codes are 32 bits:
    64 rows of 2^26 codes are not."""
    from paper_2504_03651_amd import echo
    from tests.test_fp8_host import CALL, P
    c = moe.CExperts(*{**EXPERTS, "num_experts": E, "hidden": H, "intermediate": I}.values())
    L = moe._lib()
    assert L.echo_moe_experts_workspace_bytes(ctypes.byref(c), T, top_k) == 0
    assert "intermediate" in echo.last_error()
    rc = L.echo_moe_experts(ctypes.byref(c), *{**CALL, "T": T, "top_k": top_k}.values(), P, 0, None)
    assert rc == echo.ECHO_E_UNSUPPORTED and "intermediate" in echo.last_error()
    c = moe.CExperts(*{**EXPERTS, "num_experts": E, "hidden": H, "intermediate": 1 << 23}.values())
    assert L.echo_moe_experts_workspace_bytes(ctypes.byref(c), 1, top_k) > 0
