"""Routing and experts against their fp64 references.

The chosen experts are compared exactly and the weights to a rounding of fp32
(2^-24 relative, and 1e-13 for the 64-bit scores).  An experts' output may be off by
a half step of bf16 (2^-8 relative) and what the reference allows for expert
outputs rounded to 11 bits and activation codes next to a border
(oracle/fp8_oracle.py); the error's 2-norm stays below 2^-7 of the result's.
"""
import numpy as np
import pytest

from oracle import fp8_oracle as FO
from tests.fp8_util import activations, bf16_round, dev, experts_weights
from tests.gpu_util import say

pytestmark = pytest.mark.gpu


def _route(z, kw, bias=None, bf16=False, pad=0):
    import torch
    from paper_2504_03651_amd import moe
    T, E = z.shape
    dt = torch.bfloat16 if bf16 else torch.float32
    full = torch.full((T, E + pad), float("nan"), dtype=dt, device="cuda")
    full[:, :E] = dev(z)
    k = kw["top_k"]
    ids = torch.full((T + 1, k), 77, dtype=torch.int32, device="cuda")
    w = torch.full((T + 1, k), 77.0, device="cuda")
    moe.route(moe.Router(E, **kw), full[:, :E], ids[:T], w[:T], bias=None if bias is None else dev(bias))
    torch.cuda.synchronize()
    assert (ids[T] == 77).all() and (w[T] == 77).all()
    return ids[:T].cpu().numpy(), w[:T].cpu().numpy()


def _same_route(got, want):
    assert np.array_equal(got[0], want[0]), np.argwhere(got[0] != want[0])[:4]
    # 2^-150: half of fp32's step below 2^-126, where the relative bound ends
    # (scores of a softmax over +-800 are as small as e^-250)
    assert (np.abs(got[1] - want[1]) <= (2.0 ** -24 + 1e-13) * np.abs(want[1]) + 2.0 ** -150).all()


@pytest.mark.parametrize("bf16", [False, True])
@pytest.mark.parametrize("bias", [False, True])
@pytest.mark.parametrize("T, E, kw", [
    (1, 1, dict(top_k=1)), (1, 64, dict(top_k=8)), (5, 8, dict(top_k=8, renormalize=True)),
    (33, 60, dict(top_k=4, renormalize=True, scale=2.5)), (257, 128, dict(top_k=1)),
    (70, 160, dict(top_k=6, num_groups=8, top_groups=3)),
    (70, 256, dict(top_k=8, num_groups=8, top_groups=4, group_top=2, renormalize=True)),
    (40, 512, dict(top_k=64, num_groups=64, top_groups=30, group_top=2)),
    (9, 512, dict(top_k=10, num_groups=2, top_groups=2, group_top=2)), (6, 300, dict(top_k=3)),
    (64, 16, dict(top_k=2, num_groups=16, top_groups=5))])
@pytest.mark.parametrize("score", ["softmax", "sigmoid"])
def test_route(T, E, kw, score, bias, bf16):
    g = np.random.default_rng(T + E)
    z = (2 * g.standard_normal((T, E))).astype(np.float32)
    z = bf16_round(z) if bf16 else z
    b = (0.3 * g.standard_normal(E)).astype(np.float32) if bias else None
    kw = dict(kw, score=score)
    _same_route(_route(z, kw, b, bf16, pad=T % 4), FO.route(z, bias=b, **kw))


def test_route_large_batch():
    g = np.random.default_rng(1)
    z = (1.5 * g.standard_normal((4099, 256))).astype(np.float32)
    b = (0.1 * g.standard_normal(256)).astype(np.float32)
    kw = dict(top_k=8, score="sigmoid", num_groups=8, top_groups=4, group_top=2, renormalize=True)
    _same_route(_route(z, kw, b), FO.route(z, bias=b, **kw))


@pytest.mark.parametrize("score", ["softmax", "sigmoid"])
@pytest.mark.parametrize("kw", [dict(top_k=6), dict(top_k=64),
                                dict(top_k=6, num_groups=8, top_groups=3, group_top=2),
                                dict(top_k=6, num_groups=8, top_groups=3)])
def test_route_keys_closer_than_fp32_tells(score, kw):
    """A bias that makes all keys of the first row equal but for its rounding to
    fp32, so that 64 bits decide; the rows after it differ from the first in the
    last bits of some logits, or altogether."""
    E = 128
    g = np.random.default_rng(6)
    z = np.tile(g.standard_normal(E).astype(np.float32), (40, 1))
    z[1:20] += (g.integers(-2, 3, (19, E)) * np.float32(2.0 ** -23)).astype(np.float32)
    z[20:] = g.standard_normal((20, E)).astype(np.float32)
    z64 = z[0].astype(np.float64)
    s = np.exp(z64) / np.exp(z64).sum() if score == "softmax" else 1 / (1 + np.exp(-z64))
    b = (0.75 - s).astype(np.float32)
    kw = dict(kw, score=score, renormalize=True)
    _same_route(_route(z, kw, b), FO.route(z, bias=b, **kw))


@pytest.mark.parametrize("bias", [False, True, "equal"])
@pytest.mark.parametrize("E, kw", [
    (1, dict(top_k=1)), (8, dict(top_k=2, renormalize=True)), (60, dict(top_k=15)),
    (130, dict(top_k=4, num_groups=13, top_groups=3, group_top=2, renormalize=True)),
    (160, dict(top_k=6, num_groups=16, top_groups=5)),
    (256, dict(top_k=8, num_groups=8, top_groups=4, group_top=2)),
    (512, dict(top_k=15, num_groups=2, top_groups=2, group_top=2, renormalize=True))])
@pytest.mark.parametrize("score", ["softmax", "sigmoid"])
def test_route_many_tokens(E, kw, score, bias):
    """Rows of random logits, masked ones among them, ties, and (bias "equal") rows whose
    keys are closer than fp32 tells, over and over in a batch of 4,101 tokens."""
    g = np.random.default_rng(E)
    z = (2 * g.standard_normal((37, E))).astype(np.float32)
    z[3], z[7, ::2], z[8, E // 3:], z[9] = -np.inf, -np.inf, np.nan, np.round(z[9])
    z[20:30] = z[20]
    z[21:30] += (g.integers(-2, 3, (9, E)) * np.float32(2.0 ** -23)).astype(np.float32)
    b = (0.3 * g.standard_normal(E)).astype(np.float32) if bias else None
    if bias == "equal":
        z64 = z[20].astype(np.float64)
        s = np.exp(z64) / np.exp(z64).sum() if score == "softmax" else 1 / (1 + np.exp(-z64))
        b = (0.75 - s).astype(np.float32)
    kw = dict(kw, score=score)
    ids, w = FO.route(z, bias=b, **kw)
    at = np.arange(4101) % 37
    _same_route(_route(z[at], kw, b, pad=3), (ids[at], w[at]))


@pytest.mark.parametrize("score", ["softmax", "sigmoid"])
@pytest.mark.parametrize("groups", [1, 4])
@pytest.mark.parametrize("group_top", [1, 2])
@pytest.mark.parametrize("bias", [False, True])
def test_route_ties_masks_and_extremes(score, groups, group_top, bias):
    """Equal logits, masked experts (-inf, NaN, the lowest finite value), rows that
    leave nothing or too little, infinities, and scores that saturate."""
    E = 32
    lo = float(np.finfo(np.float32).min)
    z = np.zeros((16, E), np.float32)
    z[1] = -np.inf
    z[2] = np.nan
    z[3, 3:] = -np.inf
    z[4] = lo
    z[5, ::2], z[5, 1::2] = -np.inf, 1.0
    z[6, [4, 9]] = np.inf
    z[7] = -np.inf
    z[7, 31] = np.inf
    z[8] = np.tile([90.0, -90.0, 40.0, 200.0], 8)
    z[9] = np.linspace(-800, 800, E)
    z[10, 5] = np.nan
    z[11] = np.arange(E) // 4
    z[12] = -np.arange(E) // 3
    z[13] = lo
    z[13, 7] = np.inf
    z[14, :8], z[14, 8:] = -np.inf, np.arange(24) % 5
    z[15] = np.float32(1e-30)
    b = None
    if bias:
        b = np.zeros(E, np.float32)
        b[2], b[11], b[12], b[20] = np.inf, -np.inf, np.nan, 0.5
    kw = dict(top_k=5, score=score, num_groups=groups, top_groups=min(groups, 2),
              group_top=group_top if groups > 1 else 1, renormalize=True)
    if groups == 1 and group_top == 2:
        kw.update(renormalize=False, scale=-0.5)
    got, want = _route(z, kw, b), FO.route(z, bias=b, **kw)
    _same_route(got, want)
    many = np.arange(4100) % 16
    _same_route(_route(z[many], kw, b), (want[0][many], want[1][many]))
    assert (got[0][1:3] == -1).all() and (got[1][1:3] == 0).all()


def _experts(host, ids, wt, x, xs, residual=None, in_place=False, twice=False):
    """The library's output, fp64, over a workspace of NaN bytes."""
    import torch
    from paper_2504_03651_amd import moe
    ex = moe.Experts(*[dev(a) for a in host])
    T, H = x.shape
    n = ex.workspace_bytes(T, ids.shape[1])
    full = torch.full((T + 1, H), 3.0, dtype=torch.bfloat16, device="cuda")
    out = full[:T]
    res = start = None if residual is None else dev(residual).bfloat16()
    if in_place and res is not None:
        res = out
    args = [dev(a) for a in (x, xs, ids, wt)]
    got = []
    for _ in range(2 if twice else 1):
        work = torch.full((n + 256,), 0xFF, dtype=torch.uint8, device="cuda")
        if res is out:
            out.copy_(start)
        moe.experts(ex, *args, out, work[:n], residual=res)
        torch.cuda.synchronize()
        assert (full[T] == 3.0).all() and (work[n:] == 0xFF).all()
        got.append(out.clone())
    if twice:
        assert torch.equal(got[0].view(torch.int16), got[1].view(torch.int16))
    return got[0].double().cpu().numpy()


def _near(got, want, bound):
    err = np.abs(got - want)
    assert np.isfinite(got).all()
    assert (err <= 2.0 ** -8 * np.abs(want) + bound + 2.0 ** -130).all(), float((err / (bound + 1e-30)).max())
    rel = float(np.linalg.norm(err) / max(np.linalg.norm(want), 1e-30))
    say(f"       2-norm error {rel:.2e}")
    assert rel <= 2.0 ** -7


def _routing(g, T, E, k, skew=1.0):
    z = g.standard_normal((T, E)) + skew * g.standard_normal(E)
    ids = np.argsort(-z, axis=1)[:, :k].astype(np.int32)
    return ids, g.random((T, k)).astype(np.float32)


@pytest.mark.parametrize("T, E, k, H, I", [
    (1, 1, 1, 16, 16), (1, 8, 2, 256, 128), (3, 4, 2, 144, 272), (7, 64, 8, 256, 144), (20, 3, 3, 400, 112),
    (64, 16, 2, 512, 256), (129, 8, 2, 272, 400), (300, 5, 2, 256, 384), (257, 2, 1, 1040, 128),
    (500, 4, 4, 128, 640), (40, 512, 4, 128, 48), (1000, 16, 4, 384, 256),
    # more tiles than run at once, of 16, 32, 64 and 128 pairs
    (300, 512, 4, 256, 400), (701, 512, 4, 272, 400), (401, 200, 8, 512, 400), (501, 40, 8, 1536, 1040)])
def test_experts(T, E, k, H, I):
    g = np.random.default_rng(T + E + H)
    host = experts_weights(g, E, H, I)
    x, xs = activations(g, T, H)
    ids, wt = _routing(g, T, E, k)
    say(f"[case] experts T={T} E={E} k={k} H={H} I={I}")
    r = bf16_round(g.standard_normal((T, H)).astype(np.float32)) if T % 2 else None
    want, bound = FO.experts(x, xs, ids, wt, *host, residual=r)
    _near(_experts(host, ids, wt, x, xs, r, in_place=T > 100, twice=True), want, bound)


@pytest.mark.parametrize("T", [6, 90, 700])
def test_experts_padding_repeats_and_foreign_ids(T):
    """Ids that name no expert (with any weight), an expert twice in a row, all
    tokens on one expert, rows without any: the residual, or zeros."""
    E, k, H, I = 6, 3, 256, 160
    g = np.random.default_rng(T)
    host = experts_weights(g, E, H, I)
    x, xs = activations(g, T, H)
    ids, wt = _routing(g, T, E, k)
    ids[::3] = [2, 2, 5]
    ids[1::5, 1] = -1
    ids[2::5, 0] = E
    ids[3::7] = [-1, 1 << 30, -(1 << 31)]
    wt[(ids < 0) | (ids >= E)] = np.nan
    r = bf16_round(g.standard_normal((T, H)).astype(np.float32))
    for res in (None, r):
        want, bound = FO.experts(x, xs, ids, wt, *host, residual=res)
        got = _experts(host, ids, wt, x, xs, res)
        _near(got, want, bound)
        none = ((ids < 0) | (ids >= E)).all(1)
        assert none.any() and np.array_equal(got[none], (0 * r if res is None else r)[none])
    ids[:] = 4
    wt[:] = 0.5
    want, bound = FO.experts(x, xs, ids, wt, *host)
    _near(_experts(host, ids, wt, x, xs), want, bound)
    ids[:] = -1
    assert (_experts(host, ids, wt, x, xs) == 0).all()


@pytest.mark.parametrize("T", [3, 50, 100, 700])
def test_experts_outputs_of_any_magnitude(T):
    """Columns under scales as far apart as fp32 goes, each block of them against its
    own reference; one expert's outputs are zero, and two tokens' inputs."""
    g = np.random.default_rng(T)
    E, k, H, I = 3, 2, 400, 144
    host = experts_weights(g, E, H, I)
    for b, m in enumerate((2.0 ** -118, 1.0, 2.0 ** 96, 2.0 ** -60)):
        host[3][:, b] *= np.float32(m)
    host[3][1] = 0
    x, xs = activations(g, T, H)
    x[:2] = 0
    ids, wt = _routing(g, T, E, k)
    got = _experts(host, ids, wt, x, xs)
    for b in range(4):
        at = slice(128 * b, min(128 * b + 128, H))
        want, bound = FO.experts(x, xs, ids, wt, host[0], host[1], host[2][:, at], host[3][:, b:b + 1])
        _near(got[:, at], want, bound)
    assert (got[:2] == 0).all()


def test_experts_nan_stays_in_its_token():
    g = np.random.default_rng(3)
    host = experts_weights(g, 4, 256, 256)
    x, xs = activations(g, 50, 256)
    ids, wt = _routing(g, 50, 4, 2)
    x[7, 9] = 0x7F
    xs[30, 1] = np.inf
    got = _experts(host, ids, wt, x, xs)
    bad = np.isin(np.arange(50), [7, 30])
    assert np.isnan(got[bad]).all() and np.isfinite(got[~bad]).all()


def test_experts_weights_past_32_bits():
    """The last of twenty experts whose matrices together pass 2^32 codes."""
    import torch
    from paper_2504_03651_amd import fp8, moe
    g = np.random.default_rng(2)
    E, H, I, T = 20, 8192, 14336, 3
    gu = torch.zeros(E, 2 * I, H, dtype=torch.uint8, device="cuda")
    dn = torch.zeros(E, H, I, dtype=torch.uint8, device="cuda")
    gus = torch.full((E, 2, fp8.blocks(I), fp8.blocks(H)), 2.0 ** -9, device="cuda")
    dns = torch.full((E, fp8.blocks(H), fp8.blocks(I)), 2.0 ** -9, device="cuda")
    # few values: gate and up rows 0..255 of the last expert, its down columns
    a, b = (g.integers(0, 0x78, (256, H), dtype=np.uint8) for _ in range(2))
    c = g.integers(0, 0x78, (H, 256), dtype=np.uint8)
    sgn = lambda m: m | (g.integers(0, 2, m.shape, dtype=np.uint8) << 7)   # noqa: E731
    a, b, c = sgn(a), sgn(b), sgn(c)
    gu[-1, :256], gu[-1, I:I + 256], dn[-1, :, :256] = dev(a), dev(b), dev(c)
    x, xs = activations(g, T, H)
    xs *= 2.0 ** -6
    ids, wt = np.full((T, 1), E - 1, np.int32), np.ones((T, 1), np.float32)
    ex = moe.Experts(gu, gus, dn, dns)
    out = torch.empty(T, H, dtype=torch.bfloat16, device="cuda")
    work = torch.empty(ex.workspace_bytes(T, 1), dtype=torch.uint8, device="cuda")
    moe.experts(ex, dev(x), dev(xs), dev(ids), dev(wt), out, work)
    s = lambda r, q: np.full((1, -(-r // 128), -(-q // 128)), 2.0 ** -9, np.float32)  # noqa: E731
    want, bound = FO.experts(x, xs, 0 * ids, wt, np.concatenate([a, b])[None],
                             np.stack([s(256, H), s(256, H)], 1), c[None], s(H, 256))
    _near(out.double().cpu().numpy(), want, bound)


@pytest.mark.parametrize("T", [4, 600])
def test_the_operators_together_captured_and_replayed(T):
    """Activations quantised, routed and taken through the experts, as a layer
    does: against the reference on the routing the library chose, eagerly on a
    stream of its own, and from a graph replayed over new inputs."""
    import torch
    from paper_2504_03651_amd import fp8, moe
    E, k, H, I = 16, 4, 512, 256
    g = np.random.default_rng(T)
    host = experts_weights(g, E, H, I)
    ex = moe.Experts(*[dev(a) for a in host])
    router = moe.Router(E, k, score="sigmoid", num_groups=4, top_groups=2, group_top=2, renormalize=True)
    bias = dev((0.1 * g.standard_normal(E)).astype(np.float32))
    n = ex.workspace_bytes(T, k)

    def buffers():
        e = lambda *s, t=torch.float32: torch.empty(*s, dtype=t, device="cuda")   # noqa: E731
        return dict(codes=e(T, H, t=torch.float8_e4m3fn), scales=e(T, fp8.blocks(H)),
                    ids=e(T, k, t=torch.int32), w=e(T, k), out=e(T, H, t=torch.bfloat16),
                    work=e(n, t=torch.uint8))

    x = torch.empty(T, H, dtype=torch.bfloat16, device="cuda")
    z = torch.empty(T, E, device="cuda")

    def step(b, stream=None):
        fp8.quantize(x, b["codes"], b["scales"], stream=stream)
        moe.route(router, z, b["ids"], b["w"], bias=bias, stream=stream)
        moe.experts(ex, b["codes"], b["scales"], b["ids"], b["w"], b["out"], b["work"], residual=x,
                    stream=stream)

    a, b = buffers(), buffers()
    st = torch.cuda.Stream()
    graph = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph, stream=st):
        step(a)
    for r in range(4):
        xh = bf16_round(g.standard_normal((T, H)).astype(np.float32))
        zh = g.standard_normal((T, E)).astype(np.float32)
        x.copy_(dev(xh))
        z.copy_(dev(zh))
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        step(b, stream=st)
        torch.cuda.synchronize()
        assert torch.equal(a["out"].view(torch.int16), b["out"].view(torch.int16)), r
        assert torch.equal(a["ids"], b["ids"])
    c, s = FO.quantize(xh, 1)
    ids, w = FO.route(zh, k, score="sigmoid", num_groups=4, top_groups=2, group_top=2, renormalize=True,
                      bias=bias.cpu().numpy())
    assert np.array_equal(b["ids"].cpu().numpy(), ids)
    assert np.array_equal(b["codes"].view(torch.uint8).cpu().numpy(), c)
    want, bound = FO.experts(c, s, ids, w.astype(np.float32), *host, residual=xh)
    _near(b["out"].double().cpu().numpy(), want, bound)


def test_two_calls_at_once_on_two_streams():
    import torch
    from paper_2504_03651_amd import moe
    g = np.random.default_rng(8)
    host = experts_weights(g, 8, 512, 512)
    ex = moe.Experts(*[dev(a) for a in host])
    runs = []
    for T in (200, 30):
        x, xs = activations(g, T, 512)
        ids, wt = _routing(g, T, 8, 2)
        args = [dev(a) for a in (x, xs, ids, wt)]
        new = lambda: (torch.empty(T, 512, dtype=torch.bfloat16, device="cuda"),   # noqa: E731
                       torch.empty(ex.workspace_bytes(T, 2), dtype=torch.uint8, device="cuda"))
        out, work = new()
        moe.experts(ex, *args, out, work)
        runs.append((args, out, *new(), torch.cuda.Stream()))
    torch.cuda.synchronize()
    for _ in range(20):
        for args, _, out, work, st in runs:
            moe.experts(ex, *args, out, work, stream=st)
    torch.cuda.synchronize()
    for _, want, out, _, _ in runs:
        assert torch.equal(want.view(torch.int16), out.view(torch.int16))


def test_nothing_to_do():
    import torch
    from paper_2504_03651_amd import fp8, moe
    e = lambda *s, t=torch.float32: torch.empty(*s, dtype=t, device="cuda")   # noqa: E731
    f8 = torch.float8_e4m3fn
    fp8.quantize(e(0, 256), e(0, 256, t=f8), e(0, 2))
    fp8.gemm(e(0, 256, t=f8), e(0, 2), e(64, 256, t=f8), e(1, 2), e(0, 64))
    moe.route(moe.Router(8, 2), e(0, 8), e(0, 2, t=torch.int32), e(0, 2))
    ex = moe.Experts(e(2, 64, 256, t=f8), e(2, 2, 1, 2), e(2, 256, 32, t=f8), e(2, 2, 1))
    assert ex.workspace_bytes(0, 2) == 0
    moe.experts(ex, e(0, 256, t=f8), e(0, 2), e(0, 2, t=torch.int32), e(0, 2), e(0, 256, t=torch.bfloat16),
                None)
    torch.cuda.synchronize()


def test_binding_refuses_on_the_gpu():
    import torch
    from paper_2504_03651_amd import echo, fp8
    e = lambda *s, t=torch.float32: torch.empty(*s, dtype=t, device="cuda")   # noqa: E731
    f8 = torch.float8_e4m3fn
    ok = dict(x=e(4, 256, t=f8), x_scale=e(4, 2), w=e(64, 256, t=f8), w_scale=e(1, 2), out=e(4, 64))
    for change, what in [(dict(x=e(256, 4, t=f8).t()), "not contiguous"), (dict(x_scale=e(4, 1)), "shape"),
                         (dict(w=e(64, 256)), "dtype"), (dict(out=e(64, 4).t()), "rows of out"),
                         (dict(out=e(1, 64).expand(4, 64)), "rows of out"),
                         (dict(residual=e(4, 64, t=torch.bfloat16)), "type and strides"),
                         (dict(residual=e(4, 70)[:, :64]), "type and strides")]:
        with pytest.raises(echo.EchoError, match=what):
            fp8.gemm(**{**ok, **change})
