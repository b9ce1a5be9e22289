"""The 8-bit decoder layer with experts against its fp64 reference.

Every rounding to bf16 (2^-8 at most) and to e4m3 (2^-4) is made on both sides,
of values that differ a little: a share of them falls on the other side of a
border, which moves a value by one step (2^-7, 2^-3) and is again a little
difference for the next stage.  With at most an eighth of the activations' codes
a step apart, the products' results differ by 2^-3 * sqrt(1/8) * 1/sqrt(3) = 2.5e-2
of their 2-norm (steps are spread evenly over 2^-4 .. 2^-3 of the value), the
residual stream less: the bar is 2^-5 of the output's 2-norm, and for one element
2^-3 of the largest magnitude.  A token whose last chosen expert is hardly ahead of
the next may be routed otherwise, which is no small difference: tokens nearer
than 0.02 (logits are a few 2^-8 off, times the sigmoid's slope of 1/4 at most) are
left out, and they are few.
"""
import numpy as np
import pytest

import oracle
from oracle import moe_layer_oracle as MO
from oracle.layer_oracle import bf16_value
from paper_2504_03651_amd import workload as W
from tests.gpu_util import say

pytestmark = pytest.mark.gpu

ROUTER = dict(top_k=2, score="sigmoid", num_groups=4, top_groups=2, group_top=2, renormalize=True)


def _setup(H, Hq, Hkv, D, I, E, rows):
    import torch
    from paper_2504_03651_amd import layer, moe
    lw = W.moe_layer_weights(3, H, Hq, Hkv, D, I, E)
    w = W.random_case(21, num_rows=rows, num_q_heads=Hq, num_kv_heads=Hkv, head_dim=D, max_ctx=500,
                      max_q=60)
    L = layer.MoELayer(lw, moe.Router(E, **ROUTER))
    x = W.layer_hidden(8, w.batch.num_tokens, H)
    return lw, w, L, x, torch.from_numpy(x.view(np.int16)).cuda()


@pytest.mark.parametrize("shape", [(256, 4, 2, 64, 144, 8, 6), (512, 8, 2, 128, 384, 16, 9),
                                   (1040, 4, 4, 64, 256, 8, 3)])
def test_moe_layer_matches_the_reference(shape):
    import torch
    from paper_2504_03651_amd.session import Iteration
    lw, w, L, x, hid = _setup(*shape)
    T = w.batch.num_tokens
    say(f"[case] layer with experts {shape}: {T} tokens")
    it = Iteration(w)
    ws = torch.full((L.workspace_bytes(it.pool, it.batch),), 0xFF, dtype=torch.uint8, device="cuda")
    L.forward(it.pool, it.batch, hid, ws)
    torch.cuda.synchronize()
    pool = oracle.prepare(w)
    ref, t = MO.forward(lw, ROUTER, pool, w.batch, x)
    got, want = bf16_value(hid.cpu().numpy().view(np.uint16)), bf16_value(ref)
    sure = t["distance"] > 0.02
    say(f"       {sure.sum()} of {T} tokens routed for sure")
    assert sure.mean() > 0.7
    err = np.abs(got - want)[sure]
    say(f"       2-norm error {np.linalg.norm(err) / np.linalg.norm(want[sure]):.2e}, max {err.max():.2e} "
        f"of {np.abs(want).max():.1f}")
    assert np.linalg.norm(err) <= 2.0 ** -5 * np.linalg.norm(want[sure])
    assert err.max() <= 2.0 ** -3 * np.abs(want).max()
    # the new keys: one quantisation, one product and RoPE behind the same input
    k, kr = (bf16_value(a) for a in (it.pool.k.cpu().numpy().view(np.uint16), pool.k))
    assert np.array_equal(np.isnan(k), np.isnan(kr)), "written slots differ"
    m = ~np.isnan(kr)
    assert np.linalg.norm(k[m] - kr[m]) <= 2.0 ** -5 * np.linalg.norm(kr[m])


def test_moe_layer_planned_on_the_device_and_on_another_stream():
    """Without host mirrors the results are the same within rounding; a repeated
    call on a stream of its own gives the same bits; stage times are there."""
    import torch
    from paper_2504_03651_amd import echo, layer
    from paper_2504_03651_amd.session import Iteration
    lw, w, L, x, hid = _setup(256, 4, 2, 64, 144, 8, 6)
    outs = []
    st = torch.cuda.Stream()
    for mirrors in (True, True, False):
        it = Iteration(w, mirrors=mirrors)
        h = hid.clone()
        ws = torch.empty(L.workspace_bytes(it.pool, it.batch), dtype=torch.uint8, device="cuda")
        torch.cuda.synchronize()
        was = echo.profile(True)
        L.forward(it.pool, it.batch, h, ws, stream=st)
        t = layer.timing()
        echo.profile(was)
        assert all(v > 0 for v in t.values()), t
        torch.cuda.synchronize()
        outs.append(h)
    assert torch.equal(outs[0], outs[1])
    a, b = (bf16_value(o.cpu().numpy().view(np.uint16)) for o in (outs[0], outs[2]))
    assert np.median(np.abs(a - b)) <= 2.0 ** -7 * np.abs(a).mean()
