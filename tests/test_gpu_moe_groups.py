"""Groups of experts whose sums of two keys cancel, against the fp64 reference.

With biases of opposite sign inside a group the keys are much larger than their
sum, and so is what fp32 loses of them: the sums are known to a few steps of the
keys, not of the sums.  Chosen experts are compared exactly.
"""
import numpy as np
import pytest

from oracle import fp8_oracle as FO
from tests.gpu_util import say
from tests.test_gpu_moe import _route, _same_route

pytestmark = pytest.mark.gpu


def _cancelling(g, T, E, groups, score, big):
    """(logits, bias): each group's best keys are big + p and -big + q, and the sums
    p + q of a token's groups lie 2e-6 apart in an order of its own."""
    per = E // groups
    bias = np.full((groups, per), -4 * big, np.float32)
    bias[:, 0], bias[:, 1] = big, -big
    # what a group's pair sums to, and how it is split
    step = np.argsort(g.random((T, groups)), axis=1)
    total = (0.7 if score == "sigmoid" else 0.7 / groups) * (1 + 0 * step) + 2e-6 * step
    part = total * g.uniform(0.1, 0.9, total.shape)
    p = np.full((T, groups, per), 0.3 / E)
    p[..., 0], p[..., 1] = part, total - part
    z = np.log(p / (1 - p)) if score == "sigmoid" else np.log(p)
    flip = g.random(groups) < 0.5          # the positive one is not always the first
    bias[flip, :2] = bias[flip, 1::-1]
    return z.reshape(T, E).astype(np.float32), bias.reshape(E)


@pytest.mark.parametrize("score", ["sigmoid", "softmax"])
@pytest.mark.parametrize("E, groups, top_groups, top_k", [(4, 2, 1, 2), (32, 8, 3, 5), (512, 16, 7, 9)])
@pytest.mark.parametrize("big", [2.0, 256.0, 20000.0])
def test_route_groups_whose_keys_cancel(E, groups, top_groups, top_k, score, big):
    """A few tokens and many (which take a form of their own)."""
    g = np.random.default_rng(E + int(big))
    z, b = _cancelling(g, 300, E, groups, score, big)
    kw = dict(top_k=top_k, score=score, num_groups=groups, top_groups=top_groups, group_top=2, renormalize=True)
    ids, w = FO.route(z, bias=b, **kw)
    say(f"[case] groups of cancelling keys E={E} groups={groups} {score} {big}")
    _same_route(_route(z, kw, b), (ids, w))
    at = np.arange(4500) % 300
    _same_route(_route(z[at], kw, b), (ids[at], w[at]))


@pytest.mark.parametrize("T", [1, 4097])
def test_route_two_groups_of_two(T):
    """Sums of 0.87814885 and 0.87814649, which fp32 keys near 256 put the other way."""
    z = np.tile(np.array([[0.6404342, -1.2465539, -0.07819691, -0.41511714]], np.float32), (T, 1))
    b = np.array([256, -256, 256, -256], np.float32)
    kw = dict(top_k=2, score="sigmoid", num_groups=2, top_groups=1, group_top=2)
    got = _route(z, kw, b)
    assert (got[0] == [0, 1]).all()
    _same_route(got, FO.route(z, bias=b, **kw))


def test_route_kept_groups_of_large_keys_beside_border_groups_of_small_ones():
    """The border groups' keys are small and far apart; a kept group's and a dropped
    one's cancel from 2^20 and are closer than fp32 tells."""
    g = np.random.default_rng(3)
    E, groups = 16, 4
    b = np.array([2.0 ** 20, -2.0 ** 20, -2.0 ** 23, -2.0 ** 23, 0.5, 0.5, 0.0, 0.0,
                  -0.2, -0.2, -0.9, -0.9, 2.0 ** 20, -2.0 ** 20, -2.0 ** 23, -2.0 ** 23], np.float32)
    z = g.standard_normal((200, E)).astype(np.float32)
    kw = dict(top_k=4, score="sigmoid", num_groups=groups, top_groups=2, group_top=2)
    want = FO.route(z, bias=b, **kw)
    _same_route(_route(z, kw, b), want)
    at = np.arange(4200) % 200
    _same_route(_route(z[at], kw, b), (want[0][at], want[1][at]))
