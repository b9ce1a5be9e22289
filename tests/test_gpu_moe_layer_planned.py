"""The 8-bit layer with its attention planned on the device (no host mirrors),
token by token against the fp64 reference.

The bar for a token is that of the layer's test: with at most an eighth of the
activations' codes a step apart, products differ by 2^-3 sqrt(1/8) / sqrt(3) =
2.5e-2 of their 2-norm, below 2^-5.  Tokens whose routing is decided by less than
0.02 may be routed otherwise and are left out; all of them are finite.
"""
import numpy as np
import pytest

import oracle
from oracle import moe_layer_oracle as MO
from oracle.layer_oracle import bf16_value
from tests.gpu_util import say
from tests.test_gpu_moe_layer import ROUTER, _setup

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("mirrors", [False, True])
@pytest.mark.parametrize("shape", [(256, 4, 2, 64, 144, 8, 6), (512, 8, 2, 128, 384, 16, 9)])
def test_every_token_of_the_layer(shape, mirrors):
    import torch
    from paper_2504_03651_amd.session import Iteration
    lw, w, L, x, hid = _setup(*shape)
    it = Iteration(w, mirrors=mirrors)
    ws = torch.full((L.workspace_bytes(it.pool, it.batch),), 0xFF, dtype=torch.uint8, device="cuda")
    L.forward(it.pool, it.batch, hid, ws)
    torch.cuda.synchronize()
    ref, t = MO.forward(lw, ROUTER, oracle.prepare(w), w.batch, x)
    got, want = bf16_value(hid.cpu().numpy().view(np.uint16)), bf16_value(ref)
    assert np.isfinite(got).all()
    sure = t["distance"] > 0.02
    assert sure.mean() > 0.7
    err = np.linalg.norm(got - want, axis=1) / np.linalg.norm(want, axis=1)
    say(f"[case] layer {shape} mirrors={mirrors}: {sure.sum()} tokens, worst {err[sure].max():.2e}")
    assert (err[sure] <= 2.0 ** -5).all()
