"""A workspace sized once, for the largest batch, serves every smaller one."""
import numpy as np
import pytest

from paper_2504_03651_amd import echo, fp8
from tests.gpu_util import say
from tests.test_fp8_host import GEMM, P, WSP


@pytest.mark.parametrize("N, K", [(6144, 4096), (4096, 14336), (28672, 4096), (1000, 2064), (64, 16400),
                                  (1, 16), (262288, 16384)])
def test_gemm_workspace_does_not_fall_with_the_tokens(N, K):
    need = [fp8.gemm_workspace_bytes(t, N, K) for t in range(0, 4700)]
    assert (np.diff(need) >= 0).all(), int(np.argmin(np.diff(need)))
    far = [fp8.gemm_workspace_bytes(t, N, K) for t in (4699, 10 ** 4, 10 ** 5, 10 ** 6)]
    assert sorted(far) == far and far[0] >= need[-1] and far[-1] <= 256 << 20


def test_gemm_takes_what_it_asks_for():
    """A call is refused below the bytes that were asked for, at any token count."""
    L = fp8._lib()
    for T in (1, 40, 137, 170, 196, 250, 300, 400, 2048, 4640):
        for N, K in [(6144, 4096), (4096, 14336)]:
            n = fp8.gemm_workspace_bytes(T, N, K)
            assert n > 0
            rc = L.echo_fp8_gemm(*{**GEMM, "T": T, "N": N, "K": K, "stride": N}.values(), P, n - 1, None)
            assert rc == WSP, echo.last_error()


@pytest.mark.gpu
def test_one_workspace_for_every_batch():
    """Sized for 4,640 tokens and used by the smaller batches that split K the most,
    with nothing written behind it."""
    import torch
    from oracle import fp8_oracle as FO
    from tests.fp8_util import activations, dev, weights
    g = np.random.default_rng(2)
    N, K = 768, 7168
    w, ws = weights(g, N, K)
    n = fp8.gemm_workspace_bytes(4640, N, K)
    work = torch.full((n + 256,), 0xA5, dtype=torch.uint8, device="cuda")
    wd, wsd = dev(w), dev(ws)
    for T in (1, 40, 137, 170, 250, 600):
        x, xs = activations(g, T, K)
        y = torch.empty(T, N, device="cuda")
        say(f"[case] {T} tokens in a workspace of {n} bytes")
        fp8.gemm(dev(x), dev(xs), wd, wsd, y, workspace=work[:n])
        want, S = FO.gemm(x, xs, w, ws)
        assert (np.abs(y.double().cpu().numpy() - want) <= (K + K // 128 + 4) * 2.0 ** -24 * S).all()
        assert (work[n:] == 0xA5).all()
