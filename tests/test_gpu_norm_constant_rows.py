"""Layer norms of rows of one value: the mean is that value, whatever it and the width are,
so that the norm is 0, or the bias, exactly."""
import numpy as np
import pytest

from tests.fp8_util import dev
from tests.gpu_util import say

pytestmark = pytest.mark.gpu

WIDTHS = [1, 3, 7, 9, 100, 512, 1000, 1001, 2730, 4096, 5000, 8200, 12288, 16390, 32767, 32768]


@pytest.mark.parametrize("H", WIDTHS)
def test_rows_of_one_value(H):
    import torch
    from paper_2504_03651_amd import norm
    g = np.random.default_rng(H)
    T = 200 if H <= 4096 else 40
    c = (g.standard_normal(T) * 10.0 ** g.uniform(-3, 3, T)).astype(np.float32)
    c[:3] = [100.1, 0.1, 0.0]
    x = dev(np.repeat(c[:, None], H, 1))
    say(f"[case] layer norms of rows of one value, {H}")
    b = dev(g.standard_normal(H).astype(np.float32))
    w = dev((1 + g.standard_normal(H)).astype(np.float32))
    r = dev(g.standard_normal((T, H)).astype(np.float32))
    s, y = torch.empty_like(x), torch.empty_like(x)
    norm.join(norm.Norm(H, pre="layer"), None, x, y=y)
    assert (y == 0).all()
    if H <= 16384:
        q, scale = torch.empty(T, H, dtype=torch.int8, device="cuda"), torch.empty(T, device="cuda")
        norm.join(norm.Norm(H, pre="layer"), None, x, y=q, y_scale=scale)
        assert (q == 0).all() and (scale == 1).all()
    norm.join(norm.Norm(H, pre="layer", pre_weight=w, pre_bias=b), None, x, y=y)
    assert torch.equal(y, b.expand(T, H))
    norm.join(norm.Norm(H, post="layer"), x, r, sum=s)
    assert torch.equal(s, r)
    # both norms with weights and biases: the sum's own constant
    zero = torch.zeros_like(w)
    norm.join(norm.Norm(H, post="layer", pre="layer", post_weight=w, post_bias=zero, pre_weight=w, pre_bias=b), x, x,
              sum=s, y=y)
    assert torch.equal(s, x) and torch.equal(y, b.expand(T, H))
