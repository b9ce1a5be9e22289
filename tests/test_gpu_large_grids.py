"""More rows, blocks and tokens than one launch has threads for: a launch holds fewer
than 2^32, which is 2^24 workgroups of 256."""
import pytest

from tests.gpu_util import say

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("block_rows", [1, 128])
def test_quantize_more_blocks_than_a_launch_holds(block_rows):
    """2^24 + 5 blocks of 16 values (rows of one matrix, or matrices of one row):
    powers of two, whose scale is amax / 448 and whose codes are known."""
    import torch
    from paper_2504_03651_amd import fp8
    n = 2 ** 24 + 5
    say(f"[case] quantize {n} rows in blocks of {block_rows}")
    x = torch.ones(n, 16, dtype=torch.bfloat16, device="cuda")
    x[:, 3] = 2.0 ** (torch.arange(n, device="cuda") % 7).bfloat16()
    x[:, 5] = 0
    codes = torch.full((n, 16), 0xA5, dtype=torch.uint8, device="cuda")
    scales = torch.full((n, 1), -1.0, device="cuda")
    if block_rows == 1:
        fp8.quantize(x, codes, scales)
    else:
        fp8.quantize(x.view(n, 1, 16), codes.view(n, 1, 16), scales.view(n, 1, 1), block_rows)
    want = (x.float().amax(1, keepdim=True).double() / 448).float()
    assert torch.equal(scales, want)
    # 448 / 2^j is a code: quotients of fp32 scales are within a rounding of it
    assert torch.equal(codes.view(torch.float8_e4m3fn).float(), (x.double() / want.double()).to(torch.float8_e4m3fn).float())


@pytest.mark.parametrize("T, E, kw", [(2 ** 28 + 7, 2, dict(top_k=1)),
                                      (2 ** 26 + 5, 32, dict(top_k=1, num_groups=32, top_groups=32))])
def test_route_more_tokens_than_a_launch_holds(T, E, kw):
    """A token of 16 lanes, and one of a wave: one expert ahead of equal others."""
    import torch
    from paper_2504_03651_amd import moe
    say(f"[case] route {T} tokens of {E} experts")
    at = (torch.arange(T, device="cuda", dtype=torch.int32) * 7) % E
    logits = torch.zeros(T, E, dtype=torch.bfloat16, device="cuda")
    logits.scatter_(1, at[:, None].long(), 1.0)
    ids = torch.full((T, 1), -7, dtype=torch.int32, device="cuda")
    weights = torch.full((T, 1), -1.0, device="cuda")
    moe.route(moe.Router(E, renormalize=True, **kw), logits, ids, weights)
    assert torch.equal(ids[:, 0], at) and (weights == 1).all()
