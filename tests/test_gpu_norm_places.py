"""Norms between blocks in place, and in their general forms over many rows.

In place: a row's last eight columns begin at H - 8, so that at widths that are no multiple
of eight they are read by lanes of two waves, each of which may write them only when both
have read them.  Outputs must equal, to the bit, those of the same call into buffers of
their own."""
import numpy as np
import pytest

from oracle import int8_oracle as IO
from tests.fp8_util import dev
from tests.gpu_util import say
from tests.test_gpu_norm import _case

pytestmark = pytest.mark.gpu

# where the last eight lie in two waves' columns (513: one column past 512; 1025, 2049,
# 4097 and 8193 likewise), and elsewhere; one, two and four eights a lane, 1 to 16 waves
WIDTHS = [511, 513, 519, 1001, 1025, 2049, 2730, 4097, 5001, 8193, 8201, 16383, 16390, 32767]


@pytest.mark.parametrize("kind", ["rms", "layer"])
@pytest.mark.parametrize("bf16", [True, False])
@pytest.mark.parametrize("H", WIDTHS)
def test_in_place_at_odd_widths(H, bf16, kind):
    import torch
    from paper_2504_03651_amd import norm
    g = np.random.default_rng(H)
    T, dt = 301 if H < 8000 else 101, torch.bfloat16 if bf16 else torch.float32
    say(f"[case] {kind} norms in place, {T} x {H}, bf16 {bf16}")
    new = lambda *s: dev(g.standard_normal(s).astype(np.float32)).to(dt)   # noqa: E731
    b, r, gate = new(T, H), new(T, H), new(T, H)
    usual = dict(post_weight=new(H), pre_weight=new(H))
    if kind == "layer":
        usual.update(post_bias=new(H), pre_bias=new(H))
    for more in (usual, {}):   # the usual pair, and the general form
        n = norm.Norm(H, post=kind, pre=kind, block_scale=0.5, **more)
        s, y = torch.empty_like(b), torch.empty_like(b)
        norm.join(n, b, r, gate=gate, sum=s, y=y)
        for at in ("residual", "block"):
            for out in ("sum", "y", "both"):
                x = dict(block=b.clone(), residual=r.clone())
                other = "block" if at == "residual" else "residual"
                o = dict(sum=x[at] if out != "y" else torch.empty_like(b),
                         y=x[at] if out == "y" else x[other] if out == "both" else torch.empty_like(b))
                norm.join(n, x["block"], x["residual"], gate=gate, **o)
                assert torch.equal(o["sum"], s) and torch.equal(o["y"], y), (at, out)
        if H > 16384:
            continue
        q, q2 = (torch.empty(T, H, dtype=torch.int8, device="cuda") for _ in range(2))
        z, z2 = torch.empty(T, device="cuda"), torch.empty(T, device="cuda")
        norm.join(n, b, r, gate=gate, sum=s, y=q, y_scale=z)
        for at in ("residual", "block"):
            x = dict(block=b.clone(), residual=r.clone())
            norm.join(n, x["block"], x["residual"], gate=gate, sum=x[at], y=q2, y_scale=z2)
            assert torch.equal(x[at], s) and torch.equal(q2, q) and torch.equal(z2, z), at


@pytest.mark.parametrize("stream", ["bf16", "f32"])
@pytest.mark.parametrize("H", [96, 640, 1001, 1024, 1766, 2048, 3000, 4095, 4096])
@pytest.mark.parametrize("kw", [
    dict(pre="rms", pre_weight=True), dict(pre="rms", pre_weight=True, weight_offset=1.0),
    dict(post="rms", pre="layer", post_weight=True, pre_weight=True, pre_bias=True),
    dict(post="layer", pre="rms", post_weight=True, post_bias=True, pre_weight=True),
    dict(post="rms", pre="rms", post_weight=True, pre_weight=True, weight_offset=1.0),
    dict(post="rms"), dict(pre="layer")])
def test_general_forms_of_many_rows(kw, H, stream):
    """More than 512 rows, which take fewer waves a row where y is codes."""
    g = np.random.default_rng(H)
    say(f"[case] norm of 601 x {H} into codes: {kw}, the stream in {stream}")
    _case(g, 601, H, dict(block_scale=0.22, **kw), ("bf16", stream, stream, "i8", "bf16"), pad=3 if H % 3 else 0,
          gate="channel" if H % 2 else "token")
    if "post" not in kw:
        _case(g, 601, H, kw, ("bf16", stream, stream, "i8", "bf16"), block=False)


@pytest.mark.parametrize("H", [64, 1000, 1001, 3000, 4090])
def test_an_infinite_gate_over_many_rows(H):
    """One row's scale is NaN, the others are as they were; the sum is infinite in its column
    alone."""
    import torch
    from paper_2504_03651_amd import norm
    g = np.random.default_rng(H)
    say(f"[case] an infinite gate, 601 x {H}")
    b, r, gate = (dev(g.standard_normal((601, H)).astype(np.float32)).bfloat16() for _ in range(3))
    for post in ("none", "rms"):
        n = norm.Norm(H, post=post, pre="rms")
        out = []
        for gates in (gate, gate.clone()):
            if out:
                gates[77, H - 1] = float("inf")
            s, q, z = torch.empty_like(b), torch.empty(601, H, dtype=torch.int8, device="cuda"), torch.empty(601, device="cuda")
            norm.join(n, b, r, gate=gates, sum=s, y=q, y_scale=z)
            out.append((s, q, z))
        rows = torch.arange(601, device="cuda") != 77
        for one, two in zip(*out):
            assert torch.equal(one[rows], two[rows])
        s, q, z = out[1]
        assert torch.equal(s[77, :-1], out[0][0][77, :-1]) and torch.isinf(s[77, -1])
        assert torch.isnan(z[77]) and (q[77] == 0).all()
