"""int8 quantisation and products on the GPU against the fp64 reference.

Codes and scales are compared exactly.  A product's sum is exact: fp32 results are
within the roundings that the reference counts (conversion, two scales, bias,
residual), bf16 results half a step, 2^-8 of the value, besides."""
import numpy as np
import pytest

from oracle import int8_oracle as IO
from tests.fp8_util import dev
from tests.gpu_util import say

pytestmark = pytest.mark.gpu


def _torch(a, bf16):
    import torch
    t = dev(np.asarray(a, np.float32))
    return t.to(torch.bfloat16) if bf16 else t


def _quantize(x, bf16, pad=0):
    """The codes and scales of x (values of the type), rows pad elements apart."""
    import torch
    from paper_2504_03651_amd import int8
    n, cols = x.shape
    t = _torch(x, bf16)
    if pad:
        wide = torch.full((n, cols + pad), float("nan"), dtype=t.dtype, device="cuda")
        wide[:, :cols] = t
        t = wide[:, :cols]
    codes = torch.full((n + 1, cols), 0x5A, dtype=torch.int8, device="cuda")
    scales = torch.full((n + 1,), -7.0, device="cuda")
    int8.quantize(t, codes[:n], scales[:n])
    assert (codes[n] == 0x5A).all() and scales[n] == -7   # nothing behind the last row
    return codes[:n].cpu().numpy(), scales[:n].cpu().numpy()


def _same(got, want):
    assert np.array_equal(got[1].view(np.uint32)[~np.isnan(want[1])], want[1].view(np.uint32)[~np.isnan(want[1])])
    assert np.array_equal(np.isnan(got[1]), np.isnan(want[1]))
    assert np.array_equal(got[0], want[0])


@pytest.mark.parametrize("bf16", [True, False])
@pytest.mark.parametrize("rows, cols", [(1, 16), (3, 48), (7, 512), (5, 528), (4, 1024), (3, 1040), (2, 2048),
                                        (9, 2064), (8, 4096), (3, 4112), (2, 8192), (3, 8208), (2, 14336),
                                        (2, 16384), (3, 16400), (2, 40000), (257, 272)])
def test_quantize(rows, cols, bf16):
    g = np.random.default_rng(rows * cols)
    x = (g.standard_normal((rows, cols)) * np.exp(g.standard_normal(cols))).astype(np.float32)
    x *= np.float32(2.0) ** g.integers(-20, 20, (rows, 1)).astype(np.float32)
    x = IO.bf16(x) if bf16 else x
    say(f"[case] quantize {rows} x {cols}, bf16 {bf16}")
    _same(_quantize(x, bf16, pad=0 if rows % 2 else 16), IO.quantize(x))


@pytest.mark.parametrize("bf16", [True, False])
def test_quantize_ties_and_extremes(bf16):
    """Ties at scales of powers of two and of 3; zeros, subnormal rows, the largest
    numbers, infinities and NaN."""
    import torch
    k = np.arange(-127, 127) + 0.5
    rows = []
    for s in (1.0, 2.0 ** -60, 2.0 ** 90, 2.0 ** -126, 2.0 ** -130, 2.0 ** -149, 3.0):
        rows.append(np.concatenate([k, [127.0, -127.0]]) * s)
    top = 3.3895313892515355e38   # bf16's largest
    for v in (0.0, -0.0, 2.0 ** -133, 2.0 ** -149, top, np.inf, -np.inf, np.nan):
        r = np.linspace(-1, 1, 256) * (v if np.isfinite(v) else 1.0)
        r[77] = v
        rows.append(r)
    with np.errstate(over="ignore", under="ignore"):
        x = np.array(rows).astype(np.float32)
    x = np.where(np.isfinite(x), IO.bf16(np.where(np.isfinite(x), x, 0)), x) if bf16 else x
    x = x.astype(np.float32)
    say(f"[case] quantize extremes, bf16 {bf16}")
    _same(_quantize(x, bf16), IO.quantize(x))
    wide = np.tile(x, (1, 5))     # a workgroup a row
    _same(_quantize(wide, bf16), IO.quantize(wide))
    assert torch.cuda.is_available()


def test_quantize_every_bf16_value_under_many_scales():
    """Rows whose largest magnitude runs over the significands, with every smaller
    value of eight binades below it."""
    v = np.array([(128 + m) * 2.0 ** -e for e in range(9) for m in range(128)], np.float32)
    x = np.array([np.where(v <= 128 + m, v, 0) for m in range(128)], np.float32)
    x[:, 0] = 128 + np.arange(128)
    x = np.concatenate([x, -x])
    say("[case] quantize every bf16 significand")
    _same(_quantize(x, True), IO.quantize(x))


def test_quantize_more_rows_than_a_launch_holds():
    import torch
    from paper_2504_03651_amd import int8
    n = 2 ** 25 + 5      # four rows a workgroup, 2^23 workgroups a launch
    say(f"[case] quantize {n} rows")
    x = torch.ones(n, 16, dtype=torch.bfloat16, device="cuda")
    x[:, 3] = 2.0 ** (torch.arange(n, device="cuda") % 7).bfloat16()
    codes = torch.full((n, 16), 0x5A, dtype=torch.int8, device="cuda")
    scales = torch.full((n,), -1.0, device="cuda")
    int8.quantize(x, codes, scales)
    want = (x.float().amax(1).double() / 127).float()
    assert torch.equal(scales, want)
    assert torch.equal(codes.float(), (x.double() / want.double()[:, None]).float().round())


def _operands(g, T, N, K):
    x = g.integers(-127, 128, (T, K)).astype(np.int8)
    w = np.clip(np.rint(40 * g.standard_normal((N, K))), -128, 127).astype(np.int8)
    xs = np.exp(g.standard_normal(T)).astype(np.float32) / 127
    ws = (np.exp(0.3 * g.standard_normal(N)) / np.sqrt(K) / 40).astype(np.float32)
    return x, xs, w, ws


def _gemm(x, xs, w, ws, f32, bias=None, residual=None, stride=None, in_place=False, offset=0):
    """y on the host, fp64; rows `stride` apart from element `offset` on, everything
    around them checked to be as it was."""
    import torch
    from paper_2504_03651_amd import int8
    T, N, K = len(x), len(w), x.shape[1]
    dt = torch.float32 if f32 else torch.bfloat16
    stride = N if stride is None else stride
    flat = torch.full((offset + (T + 1) * stride,), 77.0, dtype=dt, device="cuda")
    y = flat[offset:offset + T * stride].view(T, stride)[:, :N]
    res = None
    if residual is not None:
        res = y if in_place else torch.empty_like(flat)[offset:offset + T * stride].view(T, stride)[:, :N]
        res.copy_(dev(np.asarray(residual, np.float32)))
    n = int8.gemm_workspace_bytes(T, N, K)
    work = torch.full((n + 256,), 0xA5, dtype=torch.uint8, device="cuda")
    int8.gemm(dev(x), dev(xs), dev(w), dev(ws), y, bias=None if bias is None else dev(bias), residual=res,
              workspace=work[:n] if n else None)
    torch.cuda.synchronize()
    assert (work[n:] == 0xA5).all()
    got = y.double().cpu().numpy()
    y.fill_(77.0)
    assert (flat == 77.0).all(), "written beside the rows"
    return got


def _near(got, want, bound, f32):
    tol = bound + (0 if f32 else IO.BF * (np.abs(want) + bound))
    err = np.abs(got - want) - tol
    assert (err <= 0).all(), (err.max(), np.unravel_index(err.argmax(), err.shape))


SIZES = [(1, 1, 16), (1, 16, 16), (2, 17, 48), (3, 5, 144), (8, 1024, 4096), (8, 300, 14336), (9, 33, 272), (16, 100, 1040),
         (17, 260, 128), (31, 67, 2064), (32, 6000, 256), (33, 70, 2064), (48, 4096, 512), (64, 129, 8208), (65, 130, 1040),
         (67, 1000, 2064), (100, 515, 272), (128, 128, 128), (129, 257, 400), (137, 4096, 1040), (200, 300, 4112),
         (256, 256, 256), (257, 511, 384), (513, 260, 144), (1000, 3001, 272), (1031, 6150, 528)]
# each tile in one range of K and in several, the last tiles of tokens and columns cut off
SIZES += [(34, 4185, 16), (17, 1, 11296), (34, 1, 11104), (160, 6001, 4112), (35, 17615, 16), (45, 20001, 2064),
          (34, 4107, 5344), (132, 16617, 16), (132, 16617, 400), (33, 4131, 5680), (66, 16935, 16), (70, 16935, 656),
          (70, 5579, 3392), (203, 16699, 16), (203, 16699, 528), (133, 2713, 10192), (398, 16971, 16), (398, 16971, 656),
          (770, 19001, 272), (130, 10939, 8160), (97, 16894, 16), (98, 5449, 3552), (2713, 133, 7264), (161, 17594, 16),
          (164, 5685, 4880), (2012, 133, 12064), (98, 9651, 5792), (67, 2813, 9360), (2707, 145, 13856), (167, 17453, 288)]
# workgroups that go on to a next tile: more tiles than run at once
SIZES += [(40, 41003, 272), (64, 50021, 144), (190, 35003, 144), (280, 33001, 272), (1500, 8197, 144), (3001, 4099, 272),
          (900, 28679, 272), (20, 35329, 528), (259, 43662, 272), (388, 32795, 144),
          (193, 35673, 528), (258, 32974, 528), (261, 49271, 528),
          (1545, 4963, 16), (67, 16810, 4944), (193, 36583, 272)]


@pytest.mark.parametrize("f32", [True, False])
@pytest.mark.parametrize("T, N, K", SIZES)
def test_gemm(T, N, K, f32):
    g = np.random.default_rng(T * 7 + N + K)
    x, xs, w, ws = _operands(g, T, N, K)
    say(f"[case] gemm {T} x {N} x {K}, f32 {f32}")
    want, b = IO.gemm(x, xs, w, ws)
    _near(_gemm(x, xs, w, ws, f32), want, b, f32)
    # rows at odd places, bias, residual in place
    bias = g.standard_normal(N).astype(np.float32)
    res = IO.bf16(g.standard_normal((T, N)))
    want, b = IO.gemm(x, xs, w, ws, bias, res)
    _near(_gemm(x, xs, w, ws, f32, bias, res, stride=N + 3, in_place=bool(T % 2), offset=1), want, b, f32)


@pytest.mark.parametrize("T, N", [(1, 5), (40, 70), (150, 40)])
def test_gemm_sums_at_the_ends_of_32_bits(T, N):
    """The longest K with codes of -128: sums of 2^31 - 262144, and its opposite but
    for the sign of the codes that have one."""
    K = 131056
    x = np.full((T, K), -128, np.int8)
    w = np.full((N, K), -128, np.int8)
    w[1::2] = 127
    xs, ws = np.float32(2.0) ** -np.arange(T).astype(np.float32), np.ones(N, np.float32)
    say(f"[case] gemm {T} x {N} x {K}")
    want, b = IO.gemm(x, xs, w, ws)
    assert abs(want).max() == K * 16384
    _near(_gemm(x, xs, w, ws, True), want, b, True)


@pytest.mark.parametrize("T", [1, 8, 30, 64, 200, 700])
def test_gemm_scales_of_any_size(T):
    """Scales whose product, or whose product with the sum, leaves fp32 where the result
    does not; zeros, infinities and NaN stay in their rows and columns."""
    g = np.random.default_rng(T)
    N, K = 40, 144
    x, xs, w, ws = _operands(g, T, N, K)
    xs[0] = 2.0 ** 120
    ws[0], ws[1], ws[2], ws[3] = 2.0 ** -149, 2.0 ** -126, 2.0 ** 100, 2.0 ** -140
    w[4], ws[4] = 0, 2.0 ** 127
    ws[5] = 0
    if T > 1:
        xs[1] = 2.0 ** -140
    if T > 8:
        xs[2:7] = [0, np.inf, np.nan, 2.0 ** 127, 2.0 ** -149]
        ws[6:8] = [np.inf, np.nan]
    say(f"[case] gemm scales of any size, {T} tokens")
    with np.errstate(all="ignore"):
        want, b = IO.gemm(x, xs, w, ws)
        top = np.float64(np.finfo(np.float32).max)
        got = _gemm(x, xs, w, ws, True)
        out = np.abs(want) > top * (1 + 2.0 ** -25)
        assert (np.abs(got[out]) == np.inf).all() and (np.sign(got[out]) == np.sign(want[out])).all()
        assert np.array_equal(np.isnan(got), np.isnan(want))
        fine = np.abs(want) < top * (1 - 2.0 ** -20)
        assert (np.abs(got - want)[fine] <= b[fine]).all()


@pytest.mark.parametrize("N, K", [(1000, 2064), (4096, 1024), (6144, 4096)])
def test_a_tokens_results_are_the_same_in_any_batch(N, K):
    import torch
    g = np.random.default_rng(N)
    x, xs, w, ws = _operands(g, 700, N, K)
    say(f"[case] gemm batches of {N} x {K}")
    for f32 in (True, False):
        all_ = _gemm(x, xs, w, ws, f32)
        for T in (1, 8, 17, 40, 64, 100, 140, 300):
            assert np.array_equal(_gemm(x[:T], xs[:T], w, ws, f32), all_[:T]), T
    assert torch.cuda.is_available()


def test_gemm_weights_and_results_past_32_bits():
    """N * K and T * N past 2^31: one code a row is not zero."""
    import torch
    from paper_2504_03651_amd import int8
    T, N, K = 8, 2 ** 15 + 3, 2 ** 16 + 16
    say(f"[case] gemm {T} x {N} x {K}")
    w = torch.zeros(N, K, dtype=torch.int8, device="cuda")
    at = (torch.arange(N, device="cuda") * 7919) % K
    w[torch.arange(N, device="cuda"), at] = (torch.arange(N, device="cuda") % 127 + 1).to(torch.int8)
    x = torch.randint(-127, 128, (T, K), dtype=torch.int8, device="cuda")
    one = lambda n: torch.ones(n, device="cuda")   # noqa: E731
    y = torch.empty(T, N, device="cuda")
    work = torch.empty(int8.gemm_workspace_bytes(T, N, K), dtype=torch.uint8, device="cuda")
    int8.gemm(x, one(T), w, one(N), y, workspace=work)
    assert torch.equal(y, x[:, at].float() * (torch.arange(N, device="cuda") % 127 + 1).float())
    del w, work
    T, N, K = 2 ** 16 + 3, 2 ** 15 + 16, 16
    say(f"[case] gemm {T} x {N} x {K}")
    x = torch.randint(-127, 128, (T, K), dtype=torch.int8, device="cuda")
    w = torch.zeros(N, K, dtype=torch.int8, device="cuda")
    w[torch.arange(N, device="cuda"), torch.arange(N, device="cuda") % K] = 1
    y = torch.zeros(T, N, dtype=torch.bfloat16, device="cuda")
    work = torch.empty(int8.gemm_workspace_bytes(T, N, K), dtype=torch.uint8, device="cuda")
    int8.gemm(x, one(T), w, one(N), y, workspace=work)
    for t in (0, 1, 32767, 65535, 65536, T - 1):
        assert torch.equal(y[t].float(), x[t, torch.arange(N, device="cuda") % K].float()), t


def test_two_products_at_once_on_two_streams():
    import torch
    from paper_2504_03651_amd import int8
    g = np.random.default_rng(9)
    w, ws = (dev(a) for a in _operands(g, 1, 1024, 4096)[2:])
    runs = []
    for T in (137, 8, 60):
        x, xs = (dev(a) for a in _operands(g, T, 1, 4096)[:2])
        n = int8.gemm_workspace_bytes(T, 1024, 4096)
        new = lambda: (torch.empty(T, 1024, device="cuda"), torch.empty(n, dtype=torch.uint8, device="cuda"))   # noqa: E731
        y, work = new()
        int8.gemm(x, xs, w, ws, y, workspace=work)
        runs.append((x, xs, y, *new(), torch.cuda.Stream()))
    torch.cuda.synchronize()
    for _ in range(20):
        for x, xs, _, y, work, st in runs:
            int8.gemm(x, xs, w, ws, y, workspace=work, stream=st)
    torch.cuda.synchronize()
    for _, _, want, y, _, _ in runs:
        assert torch.equal(want, y)


def test_nothing_to_do():
    import torch
    from paper_2504_03651_amd import int8
    e = lambda *s, t=torch.float32: torch.empty(*s, dtype=t, device="cuda")   # noqa: E731
    i8 = torch.int8
    int8.quantize(e(0, 256), e(0, 256, t=i8), e(0))
    int8.gemm(e(0, 256, t=i8), e(0), e(64, 256, t=i8), e(64), e(0, 64))
    torch.cuda.synchronize()


def test_binding_refuses_on_the_gpu():
    import torch
    from paper_2504_03651_amd import echo, int8
    e = lambda *s, t=torch.float32: torch.empty(*s, dtype=t, device="cuda")   # noqa: E731
    i8 = torch.int8
    ok = dict(x=e(4, 256, t=i8), x_scale=e(4), w=e(64, 256, t=i8), w_scale=e(64), out=e(4, 64))
    for change, what in [(dict(x=e(256, 4, t=i8).t()), "not contiguous"), (dict(x_scale=e(4, 1)), "shape"),
                         (dict(w=e(64, 256)), "dtype"), (dict(out=e(64, 4).t()), "rows of out"),
                         (dict(out=e(1, 64).expand(4, 64)), "rows of out"), (dict(bias=e(63)), "shape"),
                         (dict(bias=e(64, t=torch.bfloat16)), "dtype"), (dict(w_scale=e(64).cpu()), "not on a GPU"),
                         (dict(residual=e(4, 64, t=torch.bfloat16)), "type and strides"),
                         (dict(residual=e(4, 70)[:, :64]), "type and strides")]:
        with pytest.raises(echo.EchoError, match=what):
            int8.gemm(**{**ok, **change})
