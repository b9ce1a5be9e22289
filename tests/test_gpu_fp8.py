"""e4m3 quantisation and products against their fp64 references.

Codes and scales are compared bit for bit.  A product's bounds, with S the sum
of the magnitudes of its terms:
  fp32 results: exact products, K + K / 128 additions and two roundings of each
    block's scale, all fp32: (K + K / 128 + 4) * 2^-24 * S;
  bf16 results: a half step of the result (2^-8 relative at most), and
    2^-12 S for the e4m3 instructions, whose sums of 128 drop what lies about 16
    bits below the largest product (2^-16 S was the most seen; a sixteenfold
    margin); the error's 2-norm stays below 2^-8 of the result's.
"""
import numpy as np
import pytest

from oracle import fp8_oracle as FO
from tests.fp8_util import activations, bf16_round, dev, weights
from tests.gpu_util import say

pytestmark = pytest.mark.gpu


def _quantize(x, dtype, block_rows, pad=0):
    """The library's codes and scales of x (fp32 values, exact in `dtype`), whose
    rows lie `pad` elements further apart; the bytes behind both stay as they were."""
    import torch
    from paper_2504_03651_amd import fp8
    t = dev(x).to(dtype)
    if pad:
        wide = torch.full((*x.shape[:-1], x.shape[-1] + pad), float("nan"), dtype=dtype, device="cuda")
        wide[..., :x.shape[-1]] = t
        t = wide[..., :x.shape[-1]]
    sshape = (*x.shape[:-2], -(-x.shape[-2] // block_rows), fp8.blocks(x.shape[-1]))
    n, m = int(np.prod(x.shape)), int(np.prod(sshape))
    codes = torch.full((n + 64,), 0xA5, dtype=torch.uint8, device="cuda")
    scales = torch.full((m + 16,), -7.0, device="cuda")
    fp8.quantize(t, codes[:n].view(*x.shape), scales[:m].view(*sshape), block_rows)
    torch.cuda.synchronize()
    assert (codes[n:] == 0xA5).all() and (scales[m:] == -7.0).all()
    return codes[:n].cpu().numpy().reshape(x.shape), scales[:m].cpu().numpy().reshape(sshape)


def _same(got, want):
    assert np.array_equal(got[1].view(np.uint32), want[1].view(np.uint32)), "scales differ"
    bad = np.argwhere(got[0] != want[0])
    assert not len(bad), (len(bad), bad[:3], got[0][tuple(bad[0])], want[0][tuple(bad[0])])


@pytest.mark.parametrize("f32", [False, True])
@pytest.mark.parametrize("block_rows", [1, 128])
@pytest.mark.parametrize("shape, pad", [((1, 16), 0), ((1, 4096), 0), ((5, 272), 16), ((129, 144), 0),
                                        ((300, 1040), 32), ((3, 130, 400), 0)])
def test_quantize(shape, pad, block_rows, f32):
    import torch
    g = np.random.default_rng(shape[-1] + block_rows)
    x = (g.standard_normal(shape) * np.exp(2 * g.standard_normal(shape))).astype(np.float32)
    say(f"[case] quantize {shape} +{pad} blocks of {block_rows} f32={f32}")
    if not f32:
        x = bf16_round(x)
    _same(_quantize(x, torch.float32 if f32 else torch.bfloat16, block_rows, pad),
          FO.quantize(x, block_rows))


def test_quantize_every_bf16_value():
    """All 2^16 bf16 patterns: NaN, infinities, subnormals and zeros beside them,
    each with ordinary neighbours and alone in a block."""
    import torch
    v = (np.arange(65536, dtype=np.uint32) << 16).view(np.float32)
    spread = np.zeros((65536, 16), np.float32)
    spread[:, 3] = v
    for x in (v.reshape(512, 128), np.random.default_rng(0).permutation(v).reshape(64, 1024), spread):
        _same(_quantize(x, torch.bfloat16, 1), FO.quantize(x, 1))
        _same(_quantize(x, torch.bfloat16, 128), FO.quantize(x, 128))


def test_quantize_fp32_edges():
    """Blocks whose scale is subnormal or underflows, ties between two codes, and
    quotients one fp32 step to either side of a tie."""
    import torch
    x = np.zeros((8, 128), np.float32)
    x[0, :3] = [1e-45, -3e-45, 1e-44]
    x[1, :4] = [1e-38, 1.1754944e-38, -5e-39, 1e-40]
    ties = (FO.TABLE[:126] + FO.TABLE[1:127]).astype(np.float32) / 2
    x[2, :126], x[2, 127] = ties, 448
    x[3, :126], x[3, 127] = np.nextafter(ties, np.float32(0)), -448
    x[4, :126], x[4, 127] = np.nextafter(ties, np.float32(1e9)), 448
    x[5, :5] = [3.4e38, -3.4e38, 1e38, 1.0, 0]
    x[6, :4] = [np.inf, 1.0, -np.inf, np.nan]
    x[7, :3] = [np.nan, np.nan, 2.0]
    for block_rows in (1, 128):
        _same(_quantize(x, torch.float32, block_rows), FO.quantize(x, block_rows))
        for r in range(8):
            _same(_quantize(x[r:r + 1], torch.float32, block_rows), FO.quantize(x[r:r + 1], block_rows))


def test_quantize_fp32_saturates_under_coarse_scales_and_keeps_infinities_apart():
    """Scales of a few subnormal steps, whose quotients pass 448 and saturate, and
    blocks with infinities and no NaN, beside ordinary blocks of the same rows."""
    import torch
    g = np.random.default_rng(4)
    x = g.standard_normal((14, 1024)).astype(np.float32)
    tiny = np.float32(2.0 ** -149)
    for r, n in enumerate([448, 627, 660, 671, 672, 1000, 1119, 1120, 1343]):
        x[r, 128:256] = 0
        x[r, 128:132] = np.array([n, -n, n // 2, 1], np.float32) * tiny
    x[9, 300], x[9, 301] = np.inf, -1.0
    x[10, 1000] = -np.inf
    x[11, 0:128] = np.inf
    x[12] *= np.float32(2.0 ** 110)
    x[13] *= np.float32(2.0 ** -110)
    for block_rows in (1, 128):
        _same(_quantize(x, torch.float32, block_rows), FO.quantize(x, block_rows))
        for r in range(14):
            _same(_quantize(x[r:r + 1], torch.float32, block_rows), FO.quantize(x[r:r + 1], block_rows))


def _gemm(x, xs, w, ws, f32, residual=None, pad=0, stream=None):
    import torch
    from paper_2504_03651_amd import fp8
    T, N, K = x.shape[0], w.shape[0], x.shape[1]
    dt = torch.float32 if f32 else torch.bfloat16
    full = torch.full((T + 1, N + pad), 3.0, dtype=dt, device="cuda")
    y = full[:T, :N]
    res = None
    if residual is not None:
        y.copy_(dev(residual))
        res = y
    n = fp8.gemm_workspace_bytes(T, N, K)
    work = torch.full((max(n, 1),), 0xFF, dtype=torch.uint8, device="cuda")
    fp8.gemm(dev(x), dev(xs), dev(w), dev(ws), y, residual=res, workspace=work if n else None)
    torch.cuda.synchronize()
    assert (full[T] == 3.0).all() and (full[:T, N:] == 3.0).all()
    return y.double().cpu().numpy()


def _check(got, want, S, K, f32):
    err = np.abs(got - want)
    if f32:
        assert (err <= (K + K // 128 + 4) * 2.0 ** -24 * S).all(), float((err / S).max())
    else:
        assert (err <= 2.0 ** -8 * np.abs(want) + 2.0 ** -12 * S).all()
        assert np.linalg.norm(err) <= 2.0 ** -8 * np.linalg.norm(want)
    return float(np.linalg.norm(err) / np.linalg.norm(want))


@pytest.mark.parametrize("f32", [False, True])
@pytest.mark.parametrize("T, N, K", [
    (1, 1, 16), (1, 100, 128), (3, 16, 144), (1, 2048, 4096), (8, 1000, 2064), (16, 257, 256),
    (17, 130, 1040), (33, 129, 640), (48, 64, 128), (64, 384, 112), (65, 100, 528), (67, 1000, 2064),
    (128, 128, 512), (129, 255, 272), (137, 512, 7168), (200, 640, 384), (256, 256, 1024),
    (257, 513, 400), (300, 1300, 2000), (513, 260, 1152), (1030, 2050, 144)])
def test_gemm(T, N, K, f32):
    g = np.random.default_rng(T * 7 + N + K)
    x, xs = activations(g, T, K)
    w, ws = weights(g, N, K)
    say(f"[case] gemm T={T} N={N} K={K} f32={f32}")
    want, S = FO.gemm(x, xs, w, ws)
    say(f"       2-norm error {_check(_gemm(x, xs, w, ws, f32, pad=T % 3), want, S, K, f32):.2e}")


@pytest.mark.parametrize("f32", [False, True])
@pytest.mark.parametrize("T, N, K", [(5, 96, 256), (70, 100, 400), (260, 300, 1280), (150, 4096, 640)])
def test_gemm_adds_the_residual_in_place(T, N, K, f32):
    g = np.random.default_rng(T)
    x, xs = activations(g, T, K)
    w, ws = weights(g, N, K)
    r = g.standard_normal((T, N)).astype(np.float32)
    r = r if f32 else bf16_round(r)
    want, S = FO.gemm(x, xs, w, ws, r)
    _check(_gemm(x, xs, w, ws, f32, r, pad=4), want, S + np.abs(r), K, f32)


@pytest.mark.parametrize("residual", [False, True])
@pytest.mark.parametrize("f32", [False, True])
@pytest.mark.parametrize("N", [63, 130, 264])
@pytest.mark.parametrize("T, K", [(5, 272), (40, 2064), (140, 4096), (300, 400)])
def test_gemm_into_columns_of_a_wider_matrix(T, N, K, f32, residual):
    """Rows of y that start at any element, what lies beside them left alone."""
    import torch
    from paper_2504_03651_amd import fp8
    g = np.random.default_rng(T + N)
    x, xs = activations(g, T, K)
    w, ws = weights(g, N, K)
    dt = torch.float32 if f32 else torch.bfloat16
    full = torch.full((T, N + 7), 3.0, dtype=dt, device="cuda")
    y = full[:, 1:N + 1]
    r = bf16_round(g.standard_normal((T, N)).astype(np.float32)) if residual else None
    if residual:
        y.copy_(dev(r))
    n = fp8.gemm_workspace_bytes(T, N, K)
    fp8.gemm(dev(x), dev(xs), dev(w), dev(ws), y, residual=y if residual else None,
             workspace=torch.empty(n, dtype=torch.uint8, device="cuda") if n else None)
    want, S = FO.gemm(x, xs, w, ws, r) if residual else FO.gemm(x, xs, w, ws)
    _check(y.double().cpu().numpy(), want, S + np.abs(r) if residual else S, K, f32)
    assert (full[:, 0] == 3.0).all() and (full[:, N + 1:] == 3.0).all()


@pytest.mark.parametrize("T", [3, 40, 300])
def test_gemm_carries_nan_and_infinity_in_their_rows_only(T):
    """A NaN code or an infinite scale of a token reaches that token alone, one of
    a weight row its own column (a weight block's scale its 128 columns)."""
    g = np.random.default_rng(T)
    x, xs = activations(g, T, 400)
    w, ws = weights(g, 300, 400)
    x[1, 77] = 0x7F
    w[290, 399] = 0xFF
    xs[2, 3] = np.inf
    got = _gemm(x, xs, w, ws, False)
    with np.errstate(all="ignore"):
        want, _ = FO.gemm(x, xs, w, ws)
    bad = np.zeros((T, 300), bool)
    bad[1], bad[:, 290], bad[2] = True, True, True
    assert not np.isfinite(got[bad]).any() and np.isfinite(got[~bad]).all()
    assert np.allclose(got[~bad], want[~bad], rtol=2.0 ** -7, atol=2.0 ** -6)


@pytest.mark.parametrize("T", [9, 400])
def test_gemm_on_another_stream_and_replayed(T):
    """The call on a stream of its own, captured, and replayed over new inputs with
    eager calls and synchronisations between the replays."""
    import torch
    from paper_2504_03651_amd import fp8
    N, K = 640, 2048
    g = np.random.default_rng(T)
    w, ws = (dev(a) for a in weights(g, N, K))
    ins = [[dev(a) for a in activations(g, T, K)] for _ in range(3)]
    x, xs = (torch.empty_like(a) for a in ins[0])
    y, eager = (torch.empty(T, N, dtype=torch.bfloat16, device="cuda") for _ in range(2))
    n = fp8.gemm_workspace_bytes(T, N, K)
    work, other = (torch.empty(max(n, 1), dtype=torch.uint8, device="cuda") for _ in range(2))
    st = torch.cuda.Stream()
    graph = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph, stream=st):
        fp8.gemm(x, xs, w, ws, y, workspace=work)
    for r in range(4):
        x.copy_(ins[r % 3][0])
        xs.copy_(ins[r % 3][1])
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        st.wait_stream(torch.cuda.current_stream())
        fp8.gemm(x, xs, w, ws, eager, workspace=other, stream=st)
        torch.cuda.synchronize()
        assert torch.equal(y.view(torch.int16), eager.view(torch.int16)), r


@pytest.mark.parametrize("T, N, K", [(20, 70001, 144), (50, 66000, 272), (100, 34008, 272),
                                     (200, 34000, 144), (700, 17000, 272), (1500, 12000, 400)])
def test_gemm_of_more_tiles_than_run_at_once(T, N, K):
    """Workgroups go from tile to tile: edges in both directions, a whole residual."""
    g = np.random.default_rng(T)
    x, xs = activations(g, T, K)
    w, ws = weights(g, N, K)
    say(f"[case] gemm T={T} N={N} K={K}")
    r = bf16_round(g.standard_normal((T, N)).astype(np.float32)) if T % 200 == 100 else None
    want, S = FO.gemm(x, xs, w, ws) if r is None else FO.gemm(x, xs, w, ws, r)
    _check(_gemm(x, xs, w, ws, False, r), want, S if r is None else S + np.abs(r), K, False)
    if T < 150:
        want, S = FO.gemm(x, xs, w, ws)
        _check(_gemm(x, xs, w, ws, True), want, S, K, True)


def test_tokens_past_32_bits():
    """More than 2^32 values quantised and codes multiplied: the first and last rows."""
    import torch
    from paper_2504_03651_amd import fp8
    g = np.random.default_rng(8)
    T, K = 262144 + 40, 16400
    a = bf16_round(g.standard_normal((2, 100, K)).astype(np.float32))
    x = torch.zeros(T, K, dtype=torch.bfloat16, device="cuda")
    x[:100], x[-100:] = dev(a[0]), dev(a[1])
    codes = torch.full((T, K), 0x55, dtype=torch.uint8, device="cuda")
    scales = torch.zeros(T, fp8.blocks(K), device="cuda")
    fp8.quantize(x, codes, scales)
    w, ws = weights(g, 40, K)
    y = torch.empty(T, 40, dtype=torch.bfloat16, device="cuda")
    n = fp8.gemm_workspace_bytes(T, 40, K)
    fp8.gemm(codes, scales, dev(w), dev(ws), y,
             workspace=torch.empty(n, dtype=torch.uint8, device="cuda") if n else None)
    for i, at in enumerate((slice(0, 100), slice(T - 100, T))):
        c, s = FO.quantize(a[i], 1)
        assert np.array_equal(codes[at].cpu().numpy(), c) and np.array_equal(scales[at].cpu().numpy(), s)
        want, S = FO.gemm(c, s, w, ws)
        _check(y[at].double().cpu().numpy(), want, S, K, False)
    assert (codes[100:-100] == 0).all() and (y[100:-100] == 0).all()


def test_gemm_offsets_past_32_bits():
    """Weights of more than 2^32 codes and outputs past 2^32 bytes: the last rows."""
    import torch
    from paper_2504_03651_amd import fp8
    g = np.random.default_rng(5)
    K, N, T = 16384, 262144 + 144, 9
    x, xs = activations(g, T, K)
    w, ws = weights(g, 272, K)
    big = torch.zeros(N, K, dtype=torch.uint8, device="cuda")
    bs = torch.ones(fp8.blocks(N), fp8.blocks(K), device="cuda")
    big[262144 - 128:] = dev(w)
    bs[2047:] = dev(ws)
    stride = 1 << 28
    flat = torch.zeros((T - 1) * stride + N, dtype=torch.bfloat16, device="cuda")
    y = torch.as_strided(flat, (T, N), (stride, 1))
    fp8.gemm(dev(x), dev(xs), big, bs, y)
    want, S = FO.gemm(x, xs, w, ws)
    _check(y[:, 262144 - 128:].double().cpu().numpy(), want, S, K, False)
    assert (y[:, :262144 - 128] == 0).all()
