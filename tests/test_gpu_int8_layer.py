"""The operators of an int8 decoder layer together, as they are used around the mixed
iteration: norm into codes, qkv product, rotary positions, append, attention, codes,
output product, both norms with gate and scaled residual, the MLP's products.

Against the fp64 reference, which makes the same roundings (bf16: 2^-8, codes: half of
amax / 127) of values that differ a little: a share of them falls on the other side of a
border and moves by one step.  With at most an eighth of the codes a step apart, steps of
1 / 127 of the largest magnitude (rows reach 3 to 4.5 times their root mean square: 0.036 of
it), the products' results differ by sqrt(1/8) * 0.036 = 1.3e-2 of their 2-norm at most; the
bar is 2^-6 of the output's 2-norm."""
import numpy as np
import pytest

import oracle
from oracle import int8_oracle as IO
from paper_2504_03651_amd import workload as W
from tests.fp8_util import dev
from tests.gpu_util import say

pytestmark = pytest.mark.gpu

H, HQ, HKV, D, R, I = 512, 8, 2, 64, 32, 1040
ROPE = dict(theta=10000.0, scaling="bands", factor=8.0, low=1.0, high=4.0, original_length=256)
FIRST = dict(pre="rms")
MID = dict(post="rms", pre="rms", residual_scale=1.0, block_scale=0.5)
LAST = dict(post="rms", residual_scale=1.0, block_scale=0.5)


def _host(g):
    w = {n: IO.quantize((g.standard_normal(s) / np.sqrt(s[1])).astype(np.float32)) for n, s in
         dict(qkv=((HQ + 2 * HKV) * D, H), o=(H, HQ * D), up=(I, H), down=(H, I)).items()}
    w["bias"] = (0.1 * g.standard_normal((HQ + 2 * HKV) * D)).astype(np.float32)
    for n in ("first", "post", "pre", "last"):
        w[n] = IO.bf16(1 + 0.2 * g.standard_normal(H))
    w["gate"] = IO.bf16(1 + 0.5 * g.standard_normal(H))
    return w


def _positions(b):
    q = np.diff(b.q_start)
    return np.concatenate([np.arange(n - c, n) for n, c in zip(b.seq_lens, q)]).astype(np.int32)


class Step:
    """Device buffers of one step and its calls."""

    def __init__(self, w, it, T):
        import torch
        from paper_2504_03651_amd import echo, int8, norm, rope
        bf, i8, f32 = torch.bfloat16, torch.int8, torch.float32
        e = lambda *s, t=bf: torch.empty(*s, dtype=t, device="cuda")   # noqa: E731
        self.it, self.T = it, T
        self.w = {n: (dev(a[0]), dev(a[1])) if isinstance(a, tuple) else dev(a) for n, a in w.items()}
        p = {n: self.w[n].to(bf) for n in ("first", "post", "pre", "last", "gate")}
        self.gate, self.bias = p["gate"], self.w["bias"]
        self.first = norm.Norm(H, pre_weight=p["first"], **FIRST)
        self.mid = norm.Norm(H, post_weight=p["post"], pre_weight=p["pre"], **MID)
        self.last = norm.Norm(H, post_weight=p["last"], **LAST)
        self.rope = rope.Rope(D, R, **ROPE)
        self.codes, self.wide, self.scale = e(T, H, t=i8), e(T, I, t=i8), e(T, t=f32)
        self.attn_codes = e(T, HQ * D, t=i8)
        self.qkv, self.q, self.k, self.v = e(T, (HQ + 2 * HKV) * D), e(T, HQ, D), e(T, HKV, D), e(T, HKV, D)
        self.attn, self.o, self.h, self.mlp, self.out, self.up = e(T, HQ, D, t=f32), e(T, H), e(T, H), e(T, H), e(T, H), e(T, I)
        n = max(int8.gemm_workspace_bytes(T, *s) for s in (((HQ + 2 * HKV) * D, H), (H, HQ * D), (I, H), (H, I)))
        self.work = torch.empty(n, dtype=torch.uint8, device="cuda")
        self.attn_ws = torch.empty(echo.workspace_bytes(it.pool, it.batch, HQ), dtype=torch.uint8, device="cuda")
        self.pos = dev(_positions(it.w.batch))

    def run(self, x, stream=None):
        import torch
        from paper_2504_03651_amd import echo, int8, norm, rope
        kw = dict(stream=stream)
        g = lambda a, s, n, y, **more: int8.gemm(a, s, *self.w[n], y, workspace=self.work, **kw, **more)   # noqa: E731
        norm.join(self.first, None, x, y=self.codes, y_scale=self.scale, **kw)
        g(self.codes, self.scale, "qkv", self.qkv, bias=self.bias)
        q, k, v = self.qkv.view(self.T, -1, D).split([HQ, HKV, HKV], 1)
        rope.rotate(self.rope, self.pos, q, k, q_out=self.q, k_out=self.k, **kw)
        with torch.cuda.stream(stream if stream is not None else torch.cuda.current_stream()):
            self.v.copy_(v)
        bits = lambda t: t.view(torch.int16)   # noqa: E731
        echo.kv_append(self.it.pool, self.it.batch, bits(self.k), bits(self.v), **kw)
        echo.attn_mixed(self.it.pool, self.it.batch, bits(self.q), HQ, D ** -0.5, self.attn, self.attn_ws, **kw)
        int8.quantize(self.attn.view(self.T, -1), self.attn_codes, self.scale, **kw)
        g(self.attn_codes, self.scale, "o", self.o)
        norm.join(self.mid, self.o, x, gate=self.gate, sum=self.h, y=self.codes, y_scale=self.scale, **kw)
        g(self.codes, self.scale, "up", self.up)
        int8.quantize(self.up, self.wide, self.scale, **kw)
        g(self.wide, self.scale, "down", self.mlp)
        norm.join(self.last, self.mlp, self.h, sum=self.out, **kw)
        return self.out


def _reference(w, wl, x, pos):
    bf = lambda a: IO.bf16(a).astype(np.float64)   # noqa: E731
    g = lambda c, n, *b: IO.gemm(*c, *w[n], *b)[0]   # noqa: E731
    c = IO.codes(IO.join(None, x, pre_weight=w["first"], **FIRST)[1][0])
    qkv = bf(g(c, "qkv", w["bias"])).reshape(len(x), -1, D)
    f, m = IO.frequencies(R, **ROPE)
    qk = bf(IO.rotate(qkv[:, :HQ + HKV], pos, f, magnitude=m)[0])
    from oracle.layer_oracle import bf16_bits
    pool = oracle.prepare(wl)
    oracle.kv_append(pool, wl.batch, bf16_bits(qk[:, HQ:]), bf16_bits(qkv[:, HQ + HKV:]))
    a = oracle.attention(pool, wl.batch, bf16_bits(qk[:, :HQ]), HQ, D ** -0.5)
    a = np.asarray(a).reshape(len(x), -1).astype(np.float32)
    o = bf(g(IO.quantize(a), "o"))
    (h, _), (y, _) = IO.join(o, x, w["gate"], post_weight=w["post"], pre_weight=w["pre"], **MID)
    up = bf(g(IO.codes(y), "up")).astype(np.float32)
    mlp = bf(g(IO.quantize(up), "down"))
    return IO.join(mlp, bf(h), post_weight=w["last"], **LAST)[0][0]


def _setup(rows=7, seed=31):
    import torch
    from paper_2504_03651_amd.session import Iteration
    g = np.random.default_rng(seed)
    wl = W.random_case(seed, num_rows=rows, num_q_heads=HQ, num_kv_heads=HKV, head_dim=D, max_ctx=300, max_q=60)
    T = wl.batch.num_tokens
    x = IO.bf16(g.standard_normal((T, H)) * np.exp(0.5 * g.standard_normal(H)))
    return _host(g), wl, T, x, Iteration(wl), dev(x).to(torch.bfloat16)


def test_the_operators_together():
    import torch
    w, wl, T, x, it, xd = _setup()
    say(f"[case] int8 layer of {T} tokens")
    got = Step(w, it, T).run(xd).double().cpu().numpy()
    want = _reference(w, wl, x, _positions(wl.batch))
    rel = np.linalg.norm(got - want) / np.linalg.norm(want)
    say(f"       2-norm error {rel:.2e}")
    assert rel <= 2.0 ** -6
    assert torch.cuda.is_available()


def test_captured_and_replayed_beside_eager_calls():
    """A graph of the step without attention's host plan (products, norms, positions),
    replayed over new inputs, beside eager calls on another stream with a workspace of
    their own; two graphs, one after the other, share one."""
    import torch
    from paper_2504_03651_amd import int8, norm, rope
    w, wl, T, x, it, xd = _setup(5, 8)
    a, b = Step(w, it, T), Step(w, it, T)

    def chain(s, stream=None):
        norm.join(s.first, None, xin, y=s.codes, y_scale=s.scale, stream=stream)
        int8.gemm(s.codes, s.scale, *s.w["qkv"], s.qkv, bias=s.bias, workspace=s.work, stream=stream)
        q, k, _ = s.qkv.view(T, -1, D).split([HQ, HKV, HKV], 1)
        rope.rotate(s.rope, s.pos, q, k, stream=stream)
        int8.quantize(s.qkv[:, :HQ * D], s.attn_codes, s.scale, stream=stream)
        int8.gemm(s.attn_codes, s.scale, *s.w["o"], s.o, workspace=s.work, stream=stream)
        norm.join(s.mid, s.o, xin, gate=s.gate, sum=s.h, y=s.codes, y_scale=s.scale, stream=stream)

    def mlp(s, stream=None):
        int8.gemm(s.codes, s.scale, *s.w["up"], s.up, workspace=s.work, stream=stream)
        int8.quantize(s.up, s.wide, s.scale, stream=stream)
        int8.gemm(s.wide, s.scale, *s.w["down"], s.out, residual=s.h, workspace=s.work, stream=stream)

    xin = torch.empty_like(xd)
    g = np.random.default_rng(3)
    st, other = torch.cuda.Stream(), torch.cuda.Stream()
    graphs = [torch.cuda.CUDAGraph(), torch.cuda.CUDAGraph()]
    torch.cuda.synchronize()
    for graph, part in zip(graphs, (chain, mlp)):
        with torch.cuda.graph(graph, stream=st):
            part(a)
    for r in range(5):
        xin.copy_(dev(IO.bf16(g.standard_normal((T, H)))))
        torch.cuda.synchronize()
        for graph in graphs:
            graph.replay()
        chain(b, other)
        mlp(b, other)
        torch.cuda.synchronize()
        for n in ("h", "codes", "wide", "out"):
            assert torch.equal(getattr(a, n), getattr(b, n)), (r, n)
