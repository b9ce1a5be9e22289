"""Sizes of the experts' workspace, and sizes that the kernels cannot address (CPU)."""
import ctypes

import numpy as np
import pytest

from paper_2504_03651_amd import moe
from tests.test_fp8_host import EXPERTS


@pytest.mark.parametrize("E, H, I", [(512, 16, 16), (512, 2048, 512), (64, 2048, 1024), (8, 4096, 14336), (1, 16, 16)])
@pytest.mark.parametrize("top_k", [1, 8])
def test_experts_workspace_does_not_fall_with_the_tokens(E, H, I, top_k):
    """Across the changes of the tiles' size, at 4, 12 and 96 pairs an expert."""
    c = moe.CExperts(*{**EXPERTS, "num_experts": E, "hidden": H, "intermediate": I}.values())
    ask = moe._lib().echo_moe_experts_workspace_bytes
    need = [ask(ctypes.byref(c), t, top_k) for t in range(0, 100 * E // top_k + 40)]
    assert (np.diff(need) >= 0).all(), int(np.argmin(np.diff(need)))
