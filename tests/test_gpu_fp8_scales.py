"""Blocks whose two scales multiply to no normal fp32 number, though what they scale
is an ordinary result: subnormal and zero products, and infinite ones.

The bounds are those of the other product tests, (K + K / 128 + 4) 2^-24 S for fp32
results and 2^-8 |y| + 2^-12 S for bf16 ones, S the sum of the terms' magnitudes, and
the share of roundings below the normal range: 2^-150 for every block's sum and the
result in fp32, 2^-134 for a bf16 result.
"""
import numpy as np
import pytest

from oracle import fp8_oracle as FO
from tests.fp8_util import activations, experts_weights, weights
from tests.gpu_util import say
from tests.test_gpu_fp8 import _gemm
from tests.test_gpu_moe import _experts, _near, _routing

pytestmark = pytest.mark.gpu


def _bounded(got, want, S, K, f32):
    err = np.abs(got - want)
    assert np.isfinite(got).all()
    if f32:
        bound = (K + K // 128 + 4) * 2.0 ** -24 * S + (K // 128 + 2) * 2.0 ** -150
    else:
        bound = 2.0 ** -8 * np.abs(want) + 2.0 ** -12 * S + 2.0 ** -134
    assert (err <= bound).all(), float((err / bound).max())


SHAPES = [(5, 300, 400), (8, 1000, 2064), (12, 257, 272), (17, 130, 1040), (33, 129, 640), (48, 64, 128),
          (67, 1000, 2064), (129, 255, 272), (137, 512, 7168), (300, 1300, 2000), (700, 17000, 272)]


@pytest.mark.parametrize("f32", [False, True])
@pytest.mark.parametrize("T, N, K", SHAPES)
def test_gemm_scales_whose_product_is_subnormal(T, N, K, f32):
    """Tokens and weight blocks of ordinary and of tiny scales (2^-62), tokens of
    large ones (2^60): tiny by tiny comes to 2^-143 to 2^-141, a few bits of fp32."""
    g = np.random.default_rng(T + N + K)
    x, xs = activations(g, T, K)
    w, ws = weights(g, N, K)
    # every scale within a factor of 2 of 2^-7 (tokens) and 2^-12 (weights)
    xs = (2.0 ** -7 * (1 + g.random(xs.shape))).astype(np.float32)
    ws = (2.0 ** -12 * (1 + g.random(ws.shape))).astype(np.float32)
    xs[::3] *= np.float32(2.0 ** -62)
    xs[1::3] *= np.float32(2.0 ** 60)
    ws[::2] *= np.float32(2.0 ** -62)
    say(f"[case] gemm T={T} N={N} K={K} f32={f32}, tiny scales")
    want, S = FO.gemm(x, xs, w, ws)
    _bounded(_gemm(x, xs, w, ws, f32), want, S, K, f32)


@pytest.mark.parametrize("f32", [False, True])
@pytest.mark.parametrize("T, N, K", SHAPES)
def test_gemm_scales_whose_product_is_infinite(T, N, K, f32):
    """Codes of the smallest values (2^-9, 2^-8) under scales that multiply to 2^130;
    single blocks of one token and of one block of rows under a scale of zero."""
    g = np.random.default_rng(T + N + K)
    x, w = (g.choice(np.array([0x00, 0x01, 0x02, 0x80, 0x81, 0x82], np.uint8), s) for s in ((T, K), (N, K)))
    x[:, 0] = w[:, 0] = 1   # no empty row
    kb = -(-K // 128)
    xs = (2.0 ** 70 * (0.5 + 0.5 * g.random((T, kb)))).astype(np.float32)
    ws = (2.0 ** 60 * (0.5 + 0.5 * g.random((-(-N // 128), kb)))).astype(np.float32)
    xs[::2] *= np.float32(2.0 ** -75)
    if kb > 1:
        xs[1, 1] = 0
        ws[-1, kb - 1] = 0
    say(f"[case] gemm T={T} N={N} K={K} f32={f32}, large scales")
    want, S = FO.gemm(x, xs, w, ws)
    assert S.max() < 2.0 ** 126
    _bounded(_gemm(x, xs, w, ws, f32), want, S, K, f32)


@pytest.mark.parametrize("f32", [False, True])
@pytest.mark.parametrize("T, N, K", SHAPES)
def test_gemm_scales_of_zero_beside_the_largest(T, N, K, f32):
    """A block under a scale of zero adds nothing, whatever the other scale and the
    block's sum: tokens of 2^120 and one of 2^-149 by rows of zero and ordinary ones."""
    g = np.random.default_rng(T * N + K)
    x, xs = activations(g, T, K)
    w, ws = weights(g, N, K)
    xs[::2, 0] = 2.0 ** 120
    xs[1, 0] = 2.0 ** -149
    ws[:, 0] = 0
    want, S = FO.gemm(x, xs, w, ws)
    _bounded(_gemm(x, xs, w, ws, f32), want, S, K, f32)


@pytest.mark.parametrize("gate, up, down", [(2.0 ** 40, 2.0 ** -77, 2.0 ** 60), (1.0, 2.0 ** -60, 2.0 ** -56)])
@pytest.mark.parametrize("T", [3, 50, 100, 700])
def test_experts_scales_whose_product_is_subnormal(T, gate, up, down):
    """The up rows' scales times the tokens' are nothing in fp32 (2^-152) under sums
    that are subnormal and large gates, or the down matrix's times the activation's are
    subnormal (2^-133); the outputs are ordinary numbers."""
    g = np.random.default_rng(T)
    E, k, H, I = 3, 2, 272, 144
    host = experts_weights(g, E, H, I)
    x, xs = activations(g, T, H)
    token = np.float32(2.0 ** -60 if down > 1 else 1)
    xs *= token
    host[1][:, 0] *= np.float32(gate) / token
    host[1][:, 1] *= np.float32(up)
    host[3][:] *= np.float32(down)
    ids, wt = _routing(g, T, E, k)
    say(f"[case] experts T={T} gate {gate} up {up} down {down}")
    want, bound = FO.experts(x, xs, ids, wt, *host)
    assert np.abs(want).max() > 2.0 ** -118
    _near(_experts(host, ids, wt, x, xs), want, bound)
