"""Rotary positions on the GPU against the fp64 reference, whose bound counts what the
angle, cos and sin, and the products in fp32 may be off; bf16 results half a step, 2^-8
of the value, besides.  Columns behind the rotary ones keep their bits."""
import numpy as np
import pytest

from oracle import int8_oracle as IO
from tests.fp8_util import dev
from tests.gpu_util import say

pytestmark = pytest.mark.gpu


def _near(got, want, bound, bf16):
    tol = bound + (IO.BF * (np.abs(want) + bound) if bf16 else 0)
    err = np.abs(got - want) - tol
    assert (err <= 0).all(), (err.max(), np.unravel_index(err.argmax(), err.shape))


def _type(bf16):
    import torch
    return torch.bfloat16 if bf16 else torch.float32


def _values(g, shape, bf16):
    x = (g.standard_normal(shape) * np.exp(g.standard_normal(shape))).astype(np.float32)
    return IO.bf16(x) if bf16 else x


CASES = [(1, 1, 1, 2, 2), (3, 2, 1, 8, 4), (5, 3, 2, 7, 4), (8, 32, 8, 128, 128), (9, 25, 5, 80, 20), (17, 4, 4, 72, 36),
         (33, 2, 2, 64, 64), (40, 8, 1, 96, 32), (7, 3, 3, 81, 80), (2, 2, 1, 1024, 1024), (3, 1, 1, 1024, 2),
         (100, 5, 5, 256, 128), (1500, 2, 1, 64, 32), (2100, 3, 1, 20, 10), (4000, 1, 1, 6, 2)]


@pytest.mark.parametrize("bf16", [True, False])
@pytest.mark.parametrize("layout", ["half", "interleaved"])
@pytest.mark.parametrize("T, hq, hkv, D, R", CASES)
def test_rotate(T, hq, hkv, D, R, layout, bf16):
    """Out of a packed projection into buffers of their own, then in place."""
    import torch
    from paper_2504_03651_amd import rope
    g = np.random.default_rng(T + D + R)
    say(f"[case] rotate {T} tokens, {hq} + {hkv} heads of {D}, {R} rotary, {layout}, bf16 {bf16}")
    r = rope.Rope(D, R, layout=layout, theta=500000.0, scaling="yarn", factor=4.0, original_length=4096)
    f, m = r.frequencies.cpu().numpy(), r.magnitude
    pos = g.integers(0, 200000, T).astype(np.int32)
    x = _values(g, (T, hq + 2 * hkv, D), bf16)
    packed = dev(x).to(_type(bf16)).view(T, -1)
    q, k = (packed[:, a * D:b * D].unflatten(1, (b - a, D)) for a, b in ((0, hq), (hq, hq + hkv)))
    qo, ko = (torch.full((T + 1, n, D), 77.0, dtype=q.dtype, device="cuda") for n in (hq, hkv))
    rope.rotate(r, dev(pos), q, k, q_out=qo[:T], k_out=ko[:T])
    want, b = IO.rotate(x, pos, f, layout, m)
    _near(qo[:T].double().cpu().numpy(), want[:, :hq], b[:, :hq], bf16)
    _near(ko[:T].double().cpu().numpy(), want[:, hq:hq + hkv], b[:, hq:hq + hkv], bf16)
    assert (qo[T] == 77).all() and (ko[T] == 77).all()
    assert np.array_equal(packed.float().cpu().numpy(), x.reshape(T, -1)), "the input changed"
    rope.rotate(r, dev(pos), q, k)
    assert torch.equal(q, qo[:T]) and torch.equal(k, ko[:T])
    assert np.array_equal(packed[:, (hq + hkv) * D:].float().cpu().numpy(), x.reshape(T, -1)[:, (hq + hkv) * D:])


@pytest.mark.parametrize("bf16", [True, False])
def test_head_major_and_odd_strides(bf16):
    """Heads before tokens, rows at odd places, one tensor alone, broadcast heads in."""
    import torch
    from paper_2504_03651_amd import rope
    g = np.random.default_rng(4)
    T, H, D = 50, 6, 48
    r = rope.Rope(D, 32, layout="interleaved")
    f = r.frequencies.cpu().numpy()
    pos = g.integers(-5000, 5000, T).astype(np.int32)
    x = _values(g, (T, H, D), bf16)
    want, b = IO.rotate(x, pos, f, "interleaved")
    say(f"[case] strides, bf16 {bf16}")
    t = dev(x).to(_type(bf16))
    flat = torch.full((3 + H * (T * 51 + 5),), 77.0, dtype=t.dtype, device="cuda")
    y = flat[3:].as_strided((T, H, D), (51, T * 51 + 5, 1), 3)
    rope.rotate(r, dev(pos), t.transpose(0, 1).contiguous().transpose(0, 1), q_out=y)
    _near(y.double().cpu().numpy(), want, b, bf16)
    y.fill_(77.0)
    assert (flat == 77.0).all()
    one = t[:, :1].expand(T, H, D)
    out = torch.empty_like(t)
    rope.rotate(r, dev(pos), one, q_out=out)
    _near(out.double().cpu().numpy(), np.repeat(want[:, :1], H, 1), np.repeat(b[:, :1], H, 1), bf16)


def test_far_positions_and_the_turn_back():
    """Positions at both ends of 32 bits; a cached key turned on by a difference, and back."""
    import torch
    from paper_2504_03651_amd import rope
    g = np.random.default_rng(5)
    D = 128
    r = rope.Rope(D, theta=10000.0)
    f = r.frequencies.cpu().numpy()
    pos = np.array([0, 1, -1, 2 ** 24 + 1, 2 ** 31 - 1, -2 ** 31, 1234567891, 2 ** 20], np.int32)
    x = _values(g, (len(pos), 2, D), False)
    say("[case] far positions")
    q = dev(x)
    rope.rotate(r, dev(pos), q)
    want, b = IO.rotate(x, pos, f)
    _near(q.double().cpu().numpy(), want, b, False)
    got = q.double().cpu().numpy()
    rope.rotate(r, dev(pos), q, inverse=True)
    back, b2 = IO.rotate(got, pos, f, inverse=True)
    _near(q.double().cpu().numpy(), back, b2, False)
    # what the turn there was off is turned back at its size
    assert np.abs(q.double().cpu().numpy() - x).max() <= (b2 + np.abs(b).max() * 2).max()
    # the gradient of a turn: against differences of the fp64 form
    u, v = g.standard_normal((1, 1, D)), g.standard_normal((1, 1, D))
    d = dev(v.astype(np.float32))
    rope.rotate(r, dev(pos[6:7]), d, inverse=True)
    e = 1e-6
    slope = [(np.sum(IO.rotate(u + e * np.eye(D)[i], pos[6:7], f)[0] * v) -
              np.sum(IO.rotate(u - e * np.eye(D)[i], pos[6:7], f)[0] * v)) / (2 * e) for i in range(D)]
    assert np.abs(d.double().cpu().numpy().ravel() - slope).max() <= 2.0 ** -18
    assert torch.cuda.is_available()


def test_frequencies_of_ones_own_infinities_and_nan():
    """Given frequencies and magnitude; NaN and infinities stay in their pairs."""
    import torch
    from paper_2504_03651_amd import rope
    g = np.random.default_rng(6)
    f = [3.0, 0.0, 1e-9, 700.25]
    r = rope.Rope(12, 8, frequencies=f, magnitude=0.5)
    x = _values(g, (4, 2, 12), False)
    pos = np.array([5, 0, 1 << 30, 77], np.int32)
    say("[case] own frequencies")
    want, b = IO.rotate(x, pos, np.array(f), magnitude=0.5)
    q = dev(x)
    q[2, 1, 3], q[1, 0, 4], q[3, 0, 9] = float("nan"), float("inf"), float("nan")
    rope.rotate(r, dev(pos), q)
    got = q.double().cpu().numpy()
    odd = np.zeros(x.shape, bool)
    odd[2, 1, [3, 7]] = odd[1, 0, [0, 4]] = odd[3, 0, 9] = True
    assert not np.isfinite(got[odd]).all() and np.isfinite(got[~odd]).all()
    assert (np.abs(got - want) <= b)[~odd].all()
    assert torch.isnan(q[3, 0, 9])


def test_more_tokens_than_a_launch_holds():
    import torch
    from paper_2504_03651_amd import rope
    T = 2 ** 24 + 2 ** 22 + 5
    say(f"[case] rotate {T} tokens")
    r = rope.Rope(512, 512, frequencies=[np.pi / 2] * 256, device="cuda")
    x = torch.zeros(T, 1, 512, dtype=torch.bfloat16, device="cuda")
    x[:, 0, 5] = 1
    pos = (torch.arange(T, device="cuda") % 4).int()
    rope.rotate(r, pos, x)
    for at, sign in ((0, (1, 0)), (1, (0, 1)), (2, (-1, 0)), (3, (0, -1))):
        a, b = x[at::4, 0, 5].float(), x[at::4, 0, 261].float()
        assert ((a - sign[0]).abs() <= 2.0 ** -20).all() and ((b - sign[1]).abs() <= 2.0 ** -20).all()
        assert x[at::4, 0, 6:261].count_nonzero() == 0


def test_no_tokens_and_refusals_on_the_gpu():
    import torch
    from paper_2504_03651_amd import echo, rope
    e = lambda *s, t=torch.float32: torch.empty(*s, dtype=t, device="cuda")   # noqa: E731
    r = rope.Rope(64)
    rope.rotate(r, e(0, t=torch.int32), e(0, 4, 64), e(0, 1, 64))
    p = e(4, t=torch.int32)
    for args, kw, what in [((p, e(4, 2, 60)), {}, "shape"), ((p.long(), e(4, 2, 64)), {}, "dtype"),
                           ((p, e(4, 2, 64), e(4, 1, 64, t=torch.bfloat16)), {}, "dtype"),
                           ((p, e(64, 2, 4).transpose(0, 2)), {}, "not adjacent"),
                           ((p, e(4, 2, 64)), dict(q_out=e(4, 3, 64)), "heads"),
                           ((p, e(4, 1, 64).expand(4, 2, 64)), {}, "overlap"),
                           ((e(5, t=torch.int32), e(4, 2, 64)), {}, "shape"), ((p, e(4, 0, 64)), {}, "heads")]:
        with pytest.raises(echo.EchoError, match=what):
            rope.rotate(r, *args, **kw)
    with pytest.raises(echo.EchoError, match="frequencies is on"):
        rope.rotate(rope.Rope(64, device="cpu"), p, e(4, 2, 64))
