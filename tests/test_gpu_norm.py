"""Norms, gate and residual between two blocks on the GPU against the fp64 reference,
whose bound follows each rounding to fp32 through both norms; bf16 results half a step,
2^-8 of the value, besides.  Codes and scales, which are decided in 64 bits, are
compared exactly."""
import numpy as np
import pytest

from oracle import int8_oracle as IO
from tests.fp8_util import dev
from tests.gpu_util import say

pytestmark = pytest.mark.gpu

WIDTHS = [1, 2, 7, 8, 9, 64, 500, 512, 513, 1000, 2048, 2049, 2730, 4096, 4100, 8192, 8200, 16384, 16390, 32768]


def _type(name):
    import torch
    return {"bf16": torch.bfloat16, "f32": torch.float32, "i8": torch.int8}[name]


def _values(a, name):
    return IO.bf16(a) if name == "bf16" else np.asarray(a, np.float32)


def _near(got, want, bound, name):
    tol = bound + (IO.BF * (np.abs(want) + bound) if name == "bf16" else 0)
    err = np.abs(got - want) - tol
    assert (err <= 0).all(), (err.max(), np.unravel_index(err.argmax(), err.shape))


def _case(g, T, H, kw, types, pad=0, gate=None, block=True, residual=True):
    """Inputs, the call, and its outputs beside the reference's."""
    import torch
    from paper_2504_03651_amd import norm
    tb, tr, ts, ty, tw = types
    x = {}
    x["block"] = _values(2 * g.standard_normal((T, H)) + 0.3, tb) if block else None
    x["residual"] = _values(3 * g.standard_normal((T, H)) - 0.2, tr) if residual else None
    x["gate"] = None if gate is None else _values(g.standard_normal((H,) if gate == "channel" else (T, H)), tb)
    w = {n: _values(1 + 0.2 * g.standard_normal(H), tw) for n in ("post_weight", "post_bias", "pre_weight", "pre_bias")
         if kw.get(n)}
    kw = {k: v for k, v in kw.items() if not k.endswith(("_weight", "_bias"))}

    def rows(a, name):
        """Rows `pad` elements apart."""
        if a is None:
            return None
        t = dev(a).to(_type(name))
        if pad and a.ndim == 2:
            wide = torch.full((len(a), H + pad), float("nan"), dtype=t.dtype, device="cuda")
            wide[:, :H] = t
            t = wide[:, :H]
        return t

    n = norm.Norm(H, **{k: dev(a).to(_type(tw)) for k, a in w.items()}, **kw)
    out = {k: torch.full((T + 1, H + pad), 77, dtype=_type(t), device="cuda") for k, t in (("sum", ts), ("y", ty)) if t}
    scale = torch.full((T + 1,), -7.0, device="cuda") if ty == "i8" else None
    norm.join(n, rows(x["block"], tb), rows(x["residual"], tr), gate=rows(x["gate"], tb),
              y_scale=None if scale is None else scale[:T], **{k: t[:T, :H] for k, t in out.items()})
    torch.cuda.synchronize()
    got = {k: t[:T, :H].clone() for k, t in out.items()}
    for t in out.values():
        t[:T, :H] = 77
        assert (t == 77).all(), "written beside the rows"
    (r, dr), (y, dy) = IO.join(x["block"], x["residual"], x["gate"], **kw, **w)
    if ts:
        _near(got["sum"].double().cpu().numpy(), r, dr, ts)
    if ty == "i8":
        codes, s = IO.codes(y)
        assert scale[T] == -7
        assert np.array_equal(scale[:T].cpu().numpy(), s)
        assert np.array_equal(got["y"].cpu().numpy(), codes)
    elif ty:
        _near(got["y"].double().cpu().numpy(), y, dy, ty)


@pytest.mark.parametrize("ty", ["bf16", "f32", "i8"])
@pytest.mark.parametrize("H", WIDTHS)
def test_both_norms(H, ty):
    if ty == "i8" and H > 16384:
        ty = "f32"     # codes are refused there
    g = np.random.default_rng(H)
    say(f"[case] norm of {H} to {ty}")
    all_ = dict(post_weight=True, post_bias=True, pre_weight=True, pre_bias=True)
    # a mean of two or fewer values leaves a layer norm nothing but its rounding
    second = "layer" if H > 2 else "rms"
    _case(g, 5, H, dict(post="rms", pre=second, post_weight=True, pre_weight=True, pre_bias=True),
          ("bf16", "bf16", "bf16", ty, "bf16"))
    _case(g, 3, H, dict(post=second, pre="rms", residual_scale=0.5, block_scale=0.22, **all_),
          ("f32", "f32", "f32", ty, "f32"), pad=3, gate="token")


@pytest.mark.parametrize("T", [1, 2, 3, 4, 5, 130])
@pytest.mark.parametrize("H", [100, 4096])
@pytest.mark.parametrize("kw, gate, block, residual", [
    (dict(pre="rms", pre_weight=True), None, False, True), (dict(post="layer"), "channel", True, False),
    (dict(post="rms", pre="rms", weight_offset=1.0, post_weight=True, pre_weight=True), None, True, True),
    (dict(residual_scale=-2.0, block_scale=0.0), "token", True, True), (dict(pre="layer", pre_bias=True), None, False, True),
    (dict(pre="rms", pre_eps=0.25), "channel", True, True)])
def test_forms(T, H, kw, gate, block, residual):
    """One input or both, every gate, no weights; sum or y alone; types mixed."""
    g = np.random.default_rng(T * H)
    say(f"[case] norm of {T} x {H}: {kw}, gate {gate}")
    for types in [("bf16", "f32", "f32", "bf16", "f32"), ("f32", "bf16", "bf16", "i8", "bf16"),
                  ("bf16", "bf16", None, "f32", "bf16"), ("bf16", "bf16", "f32", None, "f32")]:
        _case(g, T, H, kw, types, pad=5 if T % 2 else 0, gate=gate, block=block, residual=residual)


@pytest.mark.parametrize("ty", ["bf16", "i8"])
@pytest.mark.parametrize("H", [8, 9, 16, 512, 520, 1001, 2048, 2056, 2730, 4095, 4096, 4104, 8191, 8200, 16383, 16384])
@pytest.mark.parametrize("stream", ["bf16", "f32"])
@pytest.mark.parametrize("kind", ["rms", "layer"])
def test_the_usual_pairs_of_norms(H, ty, stream, kind):
    """Two RMS norms, two LAYER norms with biases; few rows and many."""
    g = np.random.default_rng(H + 1)
    say(f"[case] two {kind} norms of {H} to {ty}, the stream in {stream}")
    more = dict(post_bias=True, pre_bias=True) if kind == "layer" else {}
    for T, gate, pad in [(3, None, 0), (4, "channel", 8), (600 if H < 8200 else 520, "token", 0)]:
        _case(g, T, H, dict(post=kind, pre=kind, post_weight=True, pre_weight=True, block_scale=0.5, **more),
              ("bf16", stream, stream if T != 3 else None, ty, "bf16"), gate=gate, pad=pad)


@pytest.mark.parametrize("H", [48, 4096])
def test_in_place(H):
    import torch
    from paper_2504_03651_amd import norm
    g = np.random.default_rng(1)
    T, bf = 9, torch.bfloat16
    say(f"[case] norm in place, {H}")
    n = norm.Norm(H, post="rms", pre="layer")
    b, r = (dev(IO.bf16(g.standard_normal((T, H)))).to(bf) for _ in range(2))
    s, y = torch.empty_like(r), torch.empty_like(b)
    norm.join(n, b, r, sum=s, y=y)
    for sums, ys in ((0, 1), (1, 0)):
        buf = [b.clone(), r.clone()]
        norm.join(n, *buf, sum=buf[sums], y=buf[ys])
        assert torch.equal(buf[sums], s) and torch.equal(buf[ys], y)


@pytest.mark.parametrize("H", [64, 5000])
def test_rows_with_nothing_infinities_and_nan(H):
    """Each stays in its row: zeros (eps alone under the root), no eps, infinities, NaN,
    numbers whose squares leave fp32, tiny ones, ties of codes."""
    import torch
    from paper_2504_03651_amd import norm
    say(f"[case] norm of odd rows, {H}")
    x = np.ones((8, H), np.float32)
    x[0] = 0
    x[1, 3] = np.inf
    x[2, 5] = np.nan
    x[3] = 2.0 ** -140
    x[4, 1] = -np.inf
    x[5] = (np.arange(H) % 255 - 127) * 0.5   # codes of half steps at a scale of ...
    x[5, 0], x[6] = 127.0, (np.arange(H) % 31 - 15) * 3e30
    for pre in ("none", "rms", "layer"):
        n = norm.Norm(H, pre=pre)
        y = torch.empty(8, H, device="cuda")
        c, s = torch.empty(8, H, dtype=torch.int8, device="cuda"), torch.empty(8, device="cuda")
        norm.join(n, None, dev(x), y=y)
        norm.join(n, None, dev(x), y=c, y_scale=s)
        with np.errstate(all="ignore"):
            _, (want, b) = IO.join(None, x, pre=pre)
            codes, scales = IO.codes(want)
        got, c, s = y.double().cpu().numpy(), c.cpu().numpy(), s.cpu().numpy()
        for row in (0, 3, 5, 7):
            assert (np.abs(got[row] - want[row]) <= b[row]).all(), (pre, row)
        assert np.array_equal(s[[0, 3, 5, 6, 7]], scales[[0, 3, 5, 6, 7]]) and np.array_equal(c[[0, 3, 5, 6, 7]], codes[[0, 3, 5, 6, 7]]), pre
        for row in (1, 2, 4):
            assert np.isnan(s[row]) and (c[row] == 0).all() and not np.isfinite(got[row]).all()
        assert np.isfinite(got[7]).all()


def test_a_rows_results_are_the_same_in_any_batch():
    import torch
    from paper_2504_03651_amd import norm
    g = np.random.default_rng(3)
    for H in (200, 3000):
        b, r = (dev(g.standard_normal((3000, H)).astype(np.float32)) for _ in range(2))
        n = norm.Norm(H, post="rms", pre="rms")
        new = lambda T: (torch.empty(T, H, device="cuda"), torch.empty(T, H, device="cuda"))   # noqa: E731
        s, y = new(3000)
        norm.join(n, b, r, sum=s, y=y)
        for at, T in ((0, 1), (7, 3), (100, 1000)):
            s2, y2 = new(T)
            norm.join(n, b[at:at + T], r[at:at + T], sum=s2, y=y2)
            assert torch.equal(s2, s[at:at + T]) and torch.equal(y2, y[at:at + T])


@pytest.mark.parametrize("T, H", [(2 ** 25 + 5, 8), (2 ** 23 + 3, 520)])
def test_more_rows_than_a_launch_holds(T, H):
    import torch
    from paper_2504_03651_amd import norm
    say(f"[case] norm of {T} rows of {H}")
    x = torch.zeros(T, H, dtype=torch.bfloat16, device="cuda")
    x[:, 1] = 1 + (torch.arange(T, device="cuda") % 5).bfloat16()
    c, s = torch.full((T, H), 9, dtype=torch.int8, device="cuda"), torch.empty(T, device="cuda")
    norm.join(norm.Norm(H), None, x, y=c, y_scale=s)
    assert torch.equal(s, (x[:, 1].double() / 127).float())
    assert (c[:, 1] == 127).all() and c.count_nonzero() == T


def test_more_long_rows_than_a_launch_holds():
    """Rows of sixteen waves: 2^21 of them a launch."""
    import torch
    from paper_2504_03651_amd import norm
    T, H = 2 ** 21 + 3, 16392
    say(f"[case] norm of {T} rows of {H}")
    x = torch.zeros(T, H, dtype=torch.bfloat16, device="cuda")
    x[:, 1] = 1 + (torch.arange(T, device="cuda") % 5).bfloat16()
    norm.join(norm.Norm(H, pre="rms", pre_eps=0.0), None, x, y=x)
    # one value alone: the root of H, half a step of bf16 off
    assert ((x[:, 1].float() - H ** 0.5).abs() <= 2.0 ** -8 * H ** 0.5).all()
    for part in x.split(2 ** 16):
        assert part.count_nonzero() == len(part)
    del x, part
    torch.cuda.empty_cache()


def test_no_rows_and_refusals_on_the_gpu():
    import torch
    from paper_2504_03651_amd import echo, norm
    e = lambda *s, t=torch.float32: torch.empty(*s, dtype=t, device="cuda")   # noqa: E731
    n = norm.Norm(64, pre="rms", pre_weight=e(64))
    norm.join(n, e(0, 64), None, y=e(0, 64))
    x = e(4, 64)
    for args, kw, what in [((x, None), dict(), "neither sum nor y"), ((e(4, 60), None), dict(y=x), "shape"),
                           ((x, e(5, 64)), dict(sum=x), "shape"), ((x.half(), None), dict(y=x), "dtype"),
                           ((x, None), dict(y=e(4, 64, t=torch.int8)), "y_scale"),
                           ((x, None), dict(sum=e(4, 64, t=torch.int8)), "dtype"),
                           ((x, None), dict(y=e(64, 4).t()), "rows of y"), ((x, None), dict(y=x[:1].expand(4, 64)), "rows of y"),
                           ((x, None), dict(gate=e(63), y=x), "shape"), ((x, None), dict(sum=x, y=x), "sum is y"),
                           ((x, None), dict(y=e(4, 64, t=torch.int8), y_scale=e(3)), "shape")]:
        with pytest.raises(echo.EchoError, match=what):
            norm.join(n, *args, **kw)
    with pytest.raises(echo.EchoError, match="dtype"):
        norm.Norm(64, pre="rms", pre_weight=e(64), pre_bias=e(64, t=torch.bfloat16))
