"""Norms between blocks of rows whose squares, or whose sum, leave fp32 although the norm
does not: values up to fp32's largest, and, where eps is 0 or next to it, down to its
smallest.  Bounds are the reference's, as everywhere: a power of two that a row is held
times rounds nothing, but values 2^126 below the row's largest, of which there are none
here."""
import numpy as np
import pytest

from oracle import int8_oracle as IO
from tests.fp8_util import dev
from tests.gpu_util import say

pytestmark = pytest.mark.gpu

WIDTHS = [3, 7, 64, 1001, 2730, 4096, 8200, 12288, 16390]
TOP = float(np.finfo(np.float32).max)
BF_TOP = np.float32(2.0 ** 127 * (2 - 2.0 ** -7))


def _near(got, want, bound, bf16):
    assert np.isfinite(want).all() and np.isfinite(bound).all()
    # half a step of bf16: 2^-8 of the value, or of 2^-133, which its subnormal numbers are apart
    tol = bound + (IO.BF * (np.abs(want) + bound) + 2.0 ** -134 if bf16 else 0)
    err = np.abs(got - want) - tol
    assert (err <= 0).all(), (err.max(), np.unravel_index(err.argmax(), err.shape))


def _rows(g, H):
    """Rows of every size, ordinary ones among them."""
    x = 1.5 + g.standard_normal((11, H))
    x /= np.abs(x).max(-1, keepdims=True)
    size = np.array([1.0, 1e19, 3e19, 1e25, 3e30, 1e37, 0.999 * TOP, 1e-19, 1e-25, 1e-36, 0.5])
    return (x * size[:, None]).astype(np.float32)


@pytest.mark.parametrize("bf16", [True, False])
@pytest.mark.parametrize("eps", [1e-5, 1e-30, 0.0])
@pytest.mark.parametrize("kind", ["rms", "layer"])
@pytest.mark.parametrize("H", WIDTHS)
def test_the_second_norm(H, kind, eps, bf16):
    import torch
    from paper_2504_03651_amd import norm
    g = np.random.default_rng(H)
    x = _rows(g, H)
    if bf16:   # 0.999 of fp32's largest is an infinity there
        x = np.clip(IO.bf16(x), -BF_TOP, BF_TOP)
    say(f"[case] {kind} norm of {H} of any size, eps {eps}, bf16 {bf16}")
    dt = torch.bfloat16 if bf16 else torch.float32
    w, b = (IO.bf16(g.standard_normal(H)) for _ in range(2))
    for more in ({}, dict(pre_weight=w), dict(pre_weight=w, pre_bias=b)):
        n = norm.Norm(H, pre=kind, pre_eps=eps, **{k: dev(v).to(dt) for k, v in more.items()})
        y = torch.empty(len(x), H, dtype=dt, device="cuda")
        norm.join(n, None, dev(x).to(dt), y=y)
        _, (want, bound) = IO.join(None, x, pre=kind, pre_eps=eps, **more)
        # The product with a weight comes first.  Where that is subnormal it is half of 2^-149
        # off, which the root's reciprocal multiplies: by at most 1 / sqrt(eps), and by 2^30 at
        # most in rows that are not taken times a power of two (their mean of squares and eps
        # are at least 2^-60 together; the others' products are far from subnormal).
        if more:
            bound = bound + 2.0 ** -150 * min(2.0 ** 30, 1 / np.sqrt(eps) if eps else 2.0 ** 30)
        _near(y.double().cpu().numpy(), want, bound, bf16)


@pytest.mark.parametrize("eps", [1e-5, 0.0])
@pytest.mark.parametrize("kind", ["rms", "layer"])
@pytest.mark.parametrize("H", WIDTHS)
def test_the_first_norm(H, kind, eps):
    """Under a gate, on to an ordinary residual and a second norm: with weights and biases
    (the usual pairs), and without."""
    import torch
    from paper_2504_03651_amd import norm
    g = np.random.default_rng(H)
    x = _rows(g, H)
    r, gate = (g.standard_normal(x.shape).astype(np.float32) for _ in range(2))
    say(f"[case] {kind} norm of {H} of any size behind a block, eps {eps}")
    names = ["post_weight", "pre_weight"] + (["post_bias", "pre_bias"] if kind == "layer" else [])
    w = {n: (1 + 0.2 * g.standard_normal(H)).astype(np.float32) for n in names}
    for more in ({}, w):
        n = norm.Norm(H, post=kind, pre=kind, post_eps=eps, **{k: dev(v) for k, v in more.items()})
        s, y = torch.empty(x.shape, device="cuda"), torch.empty(x.shape, device="cuda")
        norm.join(n, dev(x), dev(r), gate=dev(gate), sum=s, y=y)
        (want, bound), (ywant, ybound) = IO.join(x, r, gate, post=kind, pre=kind, post_eps=eps, **more)
        _near(s.double().cpu().numpy(), want, bound, False)
        _near(y.double().cpu().numpy(), ywant, ybound, False)


@pytest.mark.parametrize("H", [64, 5000])
def test_numbers_whose_squares_leave_fp32(H):
    import torch
    from paper_2504_03651_amd import norm
    x = ((np.arange(H) % 31 - 15) * 3e30).astype(np.float32)[None]
    say(f"[case] squares that leave fp32, {H}")
    for pre in ("rms", "layer"):
        y = torch.empty(1, H, device="cuda")
        norm.join(norm.Norm(H, pre=pre), None, dev(x), y=y)
        _, (want, bound) = IO.join(None, x, pre=pre)
        _near(y.double().cpu().numpy(), want, bound, False)


@pytest.mark.parametrize("H", [3, 1000, 4100])
def test_rows_of_one_value_of_any_size(H):
    """The largest and the smallest numbers, all alike: a layer norm leaves 0, under any
    eps above 0; an RMS norm without eps 1."""
    import torch
    from paper_2504_03651_amd import norm
    c = np.array([TOP, -TOP, 2.0 ** 127, 2.0 ** 100, 2.0 ** -100, 2.0 ** -126, 2.0 ** -149, -1.0], np.float32)
    x = np.repeat(c[:, None], H, 1)
    say(f"[case] rows of one value, {H}")
    y = torch.empty(x.shape, device="cuda")
    for eps in (1e-5, 1e-38):
        norm.join(norm.Norm(H, pre="layer", pre_eps=eps), None, dev(x), y=y)
        assert (y == 0).all()
    norm.join(norm.Norm(H, pre="rms", pre_eps=0.0), None, dev(x), y=y)
    # sums of up to 12 and 33 values in a lane and between lanes, a root, three products
    assert ((y.cpu() - torch.from_numpy(np.sign(x))).abs() <= 64 * IO.U).all()
