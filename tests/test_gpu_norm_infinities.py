"""An infinity in a row of the norms between blocks: where the root of the squares' mean is
infinite the row's norm is 0, and NaN in the infinity's own column.  That holds wherever
the infinity stands: the last eight columns are held by more lanes than one, or by lanes
behind the row's end as well, and count once."""
import numpy as np
import pytest

from oracle import int8_oracle as IO
from tests.fp8_util import dev
from tests.gpu_util import say

pytestmark = pytest.mark.gpu

WIDTHS = [2, 7, 9, 64, 1000, 1001, 2048, 2049, 2730, 4100, 5120, 8200, 16383]


def _join(x, H, kw, ty, T):
    """(sum, y, scales) on the host."""
    import torch
    from paper_2504_03651_amd import norm
    f32 = torch.float32
    tys = {"bf16": torch.bfloat16, "f32": f32, "i8": torch.int8}
    n = norm.Norm(H, **{k: dev(v) if k.endswith("weight") else v for k, v in kw.items()})
    s, y = torch.empty(T, H, dtype=f32, device="cuda"), torch.empty(T, H, dtype=tys[ty], device="cuda")
    scale = torch.empty(T, device="cuda") if ty == "i8" else None
    norm.join(n, dev(x["block"]), dev(x["residual"]), gate=dev(x["gate"]), sum=s, y=y, y_scale=scale)
    return s.cpu().numpy(), y.float().cpu().numpy(), None if scale is None else scale.cpu().numpy()


@pytest.mark.parametrize("ty", ["bf16", "f32"])
@pytest.mark.parametrize("post", ["none", "rms"])
@pytest.mark.parametrize("H", WIDTHS)
def test_infinities_before_the_second_norm(H, post, ty):
    """In the residual, in the gate, in the block (under no norm), in the first norm's weight:
    one column of the sum."""
    g = np.random.default_rng(H)
    T, hit = 5, 2
    w = {"pre_weight": (1 + 0.2 * g.standard_normal(H)).astype(np.float32)}
    if post == "rms":
        w["post_weight"] = (1 + 0.2 * g.standard_normal(H)).astype(np.float32)
    x = {n: IO.bf16(g.standard_normal((T, H))) for n in ("block", "residual", "gate")}
    kw = dict(post=post, pre="rms", **w)
    s0, y0, _ = _join(x, H, kw, ty, T)
    assert np.isfinite(s0).all() and np.isfinite(y0).all()
    for at in sorted({0, H // 2, max(H - 5, 0), H - 1}):
        for where in ("residual", "gate", "post_weight" if post == "rms" else "block"):
            say(f"[case] an infinity in {where}, column {at} of {H}, {post} before, to {ty}")
            x1, kw1, rows = {n: v.copy() for n, v in x.items()}, dict(kw), np.arange(T) == hit
            if where == "post_weight":
                kw1[where] = w[where].copy()
                kw1[where][at] = np.inf
                rows[:] = True
            else:
                x1[where][hit, at] = np.inf
            s, y, _ = _join(x1, H, kw1, ty, T)
            cols = np.arange(H) == at
            assert np.array_equal(s[~rows], s0[~rows]) and np.array_equal(y[~rows], y0[~rows])
            assert np.array_equal(s[rows][:, ~cols], s0[rows][:, ~cols]) and np.isinf(s[rows][:, cols]).all()
            assert (y[rows][:, ~cols] == 0).all() and np.isnan(y[rows][:, cols]).all()


@pytest.mark.parametrize("ty", ["bf16", "f32", "i8"])
@pytest.mark.parametrize("weights", [True, False])
@pytest.mark.parametrize("H", WIDTHS)
def test_infinities_before_the_first_norm(H, weights, ty):
    """The block's norm is 0 but for one column: the sum is the residual there."""
    g = np.random.default_rng(H)
    T, hit = 5, 2
    x = {n: IO.bf16(g.standard_normal((T, H))) for n in ("block", "residual", "gate")}
    kw = dict(post="rms", pre="rms")
    if weights:
        kw.update({n: (1 + 0.2 * g.standard_normal(H)).astype(np.float32) for n in ("post_weight", "pre_weight")})
    s0, y0, q0 = _join(x, H, kw, ty, T)
    rows = np.arange(T) == hit
    for at in sorted({0, max(H - 5, 0), H - 1}):
        say(f"[case] an infinity in the block, column {at} of {H}, to {ty}")
        x1 = {n: v.copy() for n, v in x.items()}
        x1["block"][hit, at] = -np.inf
        s, y, q = _join(x1, H, kw, ty, T)
        cols = np.arange(H) == at
        assert np.array_equal(s[~rows], s0[~rows]) and np.array_equal(y[~rows], y0[~rows])
        assert np.array_equal(s[hit, ~cols], x["residual"][hit, ~cols]) and np.isnan(s[hit, at])
        if ty == "i8":
            assert np.isnan(q[hit]) and (y[hit] == 0).all() and np.array_equal(q[~rows], q0[~rows])
        else:
            assert np.isnan(y[hit]).all()
