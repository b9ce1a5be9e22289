"""How far products and experts are from 64 bits in the 2-norm.

Roundings to bf16 are spread evenly over half a step, 2^-8 of the power of two below
the value: their mean square is at most (2^-8)^2 / 3 of it, 2.26e-3 in the 2-norm,
the products' whole bar with 3% to spare (the e4m3 sums' 1.5e-5 is nothing beside it).
An expert's activation has codes a step of 2^-4 to 2^-3 apart, and sums behind them
that are sqrt(2) 1.5e-5, with the gate's slope up to 3e-5, off: a share of 0.8 x 3e-5 /
step of the codes is one step away, whose mean square is 0.8 x 3e-5 x 0.09 = 2.2e-6
of theirs, 1.5e-3 in the 2-norm.  With the output's rounding to 11 bits (2.8e-4) and
the result's to bf16 that is 2.7e-3; the bar is 3e-3.
"""
import numpy as np
import pytest

from oracle import fp8_oracle as FO
from tests.fp8_util import activations, experts_weights, weights
from tests.gpu_util import say
from tests.test_gpu_fp8 import _gemm
from tests.test_gpu_moe import _experts, _routing

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("T, N, K", [(8, 12000, 2048), (32, 4000, 1040), (64, 2048, 4096), (137, 1024, 7168),
                                     (600, 2050, 1024)])
def test_products(T, N, K):
    g = np.random.default_rng(T)
    x, xs = activations(g, T, K)
    w, ws = weights(g, N, K)
    want, _ = FO.gemm(x, xs, w, ws)
    rel = np.linalg.norm(_gemm(x, xs, w, ws, False) - want) / np.linalg.norm(want)
    say(f"[case] gemm {T} x {N} x {K}: {rel:.2e}")
    assert rel <= 1.03 * 2.0 ** -8 / np.sqrt(3)


@pytest.mark.parametrize("T, E, k, H, I", [(24, 16, 2, 2048, 512), (60, 8, 1, 2048, 512), (200, 8, 2, 1024, 640),
                                           (700, 8, 2, 1024, 512)])
def test_experts(T, E, k, H, I):
    """Tiles of 16, 32, 64 and 128 pairs."""
    g = np.random.default_rng(T)
    host = experts_weights(g, E, H, I)
    x, xs = activations(g, T, H)
    ids, wt = _routing(g, T, E, k)
    want, _ = FO.experts(x, xs, ids, wt, *host)
    rel = np.linalg.norm(_experts(host, ids, wt, x, xs) - want) / np.linalg.norm(want)
    say(f"[case] experts {T} tokens, {E} experts: {rel:.2e}")
    assert rel <= 3e-3
