"""Products in 8-bit integers in every cut: each form of the kernels in each number of
ranges of K against the definition in 64 bits (bounds as in the reference: a rounding each
for the sum's conversion, the two scales, bias and residual; bf16 half a step besides),
batches whose cuts differ to the bit, and the ranges' sums in workspaces that are shared or
used at once."""
import numpy as np
import pytest

from oracle import int8_oracle as IO
from tests import int8_sizes as S
from tests.gpu_util import say

pytestmark = pytest.mark.gpu


def _operands(seed, T, N, K):
    """Codes, scales, bias and residual on the GPU."""
    import torch
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    new = lambda *s: torch.randn(*s, generator=g, device="cuda")   # noqa: E731
    x = torch.randint(-127, 128, (T, K), generator=g, dtype=torch.int8, device="cuda")
    w = torch.randint(-128, 128, (N, K), generator=g, dtype=torch.int8, device="cuda")
    xs, ws = new(T).exp() / 127, (0.3 * new(N)).exp() / (40 * K ** 0.5)
    return x, xs, w, ws, new(N), new(T, N).bfloat16()


def _work(T, N, K):
    import torch
    from paper_2504_03651_amd import int8
    return torch.empty(int8.gemm_workspace_bytes(T, N, K), dtype=torch.uint8, device="cuda")


@pytest.mark.parametrize("T, N, K, f32", S.FORMS)
def test_every_form(T, N, K, f32):
    """With a bias and a residual in place, in rows at odd places; nothing beside them is
    written."""
    import torch
    from paper_2504_03651_amd import int8
    say(f"[case] gemm {T} x {N} x {K}, f32 {f32}")
    x, xs, w, ws, bias, res = _operands(T + N + K, T, N, K)
    dt = torch.float32 if f32 else torch.bfloat16
    stride = N + 5
    flat = torch.full((1 + (T + 1) * stride,), 77.0, dtype=dt, device="cuda")
    y = flat[1:1 + T * stride].view(T, stride)[:, :N]
    y.copy_(res)
    n = int8.gemm_workspace_bytes(T, N, K)
    work = torch.full((n + 256,), 0xA5, dtype=torch.uint8, device="cuda")
    int8.gemm(x, xs, w, ws, y, bias=bias, residual=y, workspace=work[:n] if n else None)
    xd = x.double()
    for i in range(0, N, 2048):
        at = slice(i, i + 2048)
        v = (xd @ w[at].double().t().contiguous()) * xs.double()[:, None] * ws[at].double()
        tol = 3 * IO.U * v.abs()
        for more in (bias[at].double(), res[:, at].double()):
            v = v + more
            tol = tol + IO.U * v.abs()
        tol = tol * (1 + 2.0 ** -20)
        if not f32:
            tol = tol + IO.BF * (v.abs() + tol)
        assert ((y[:, at].double() - v).abs() <= tol).all(), i
    assert (work[n:] == 0xA5).all()
    y.fill_(77.0)
    assert (flat == 77.0).all(), "written beside the rows"


@pytest.mark.parametrize("f32", [True, False])
@pytest.mark.parametrize("N, K", S.WEIGHTS)
def test_a_tokens_results_are_the_same_under_any_cut(N, K, f32):
    import torch
    from paper_2504_03651_amd import int8
    say(f"[case] batches of {N} x {K}, f32 {f32}")
    most = max(S.BATCHES)
    x, xs, w, ws, bias, res = _operands(N, most, N, K)
    dt = torch.float32 if f32 else torch.bfloat16
    work = _work(most, N, K)   # serves every smaller batch
    ys = []
    for T in S.BATCHES:
        y = torch.full((T, N), 77.0, dtype=dt, device="cuda")
        int8.gemm(x[:T], xs[:T], w, ws, y, bias=bias, residual=res[:T].to(dt), workspace=work)
        ys.append(y)
    for T, y in zip(S.BATCHES, ys):
        assert torch.equal(y, ys[-1][:T]), T


def test_products_in_ranges_at_once_on_streams():
    """Each with a workspace of its own, over and over on a stream of its own."""
    import torch
    from paper_2504_03651_amd import int8
    runs = []
    for i, (T, N, K) in enumerate(S.STREAMS):
        x, xs, w, ws, bias, _ = _operands(i, T, N, K)
        want, y = (torch.empty(T, N, device="cuda") for _ in range(2))
        work = _work(T, N, K)
        int8.gemm(x, xs, w, ws, want, bias=bias, workspace=work)
        runs.append((x, xs, w, ws, bias, want, y, _work(T, N, K), torch.cuda.Stream()))
    torch.cuda.synchronize()
    for _ in range(20):
        for x, xs, w, ws, bias, _, y, work, st in runs:
            int8.gemm(x, xs, w, ws, y, bias=bias, workspace=work, stream=st)
    torch.cuda.synchronize()
    for *_, want, y, _, _ in runs:
        assert torch.equal(want, y)


def test_graphs_that_share_a_workspace_beside_eager_calls():
    """Two graphs of a product in ranges each, one after the other over one workspace, with
    new inputs at each replay; eager calls of the same products, with another workspace, on
    another stream meanwhile."""
    import torch
    from paper_2504_03651_amd import int8
    ops = [_operands(i, *s) for i, s in enumerate(S.GRAPHS)]
    work, other = (torch.empty(max(_work(*s).numel() for s in S.GRAPHS), dtype=torch.uint8, device="cuda")
                   for _ in range(2))
    ys, eager = ([torch.empty(T, N, device="cuda") for T, N, _ in S.GRAPHS] for _ in range(2))

    def product(i, y, space, stream=None):
        x, xs, w, ws, bias, _ = ops[i]
        int8.gemm(x, xs, w, ws, y, bias=bias, workspace=space, stream=stream)

    st, aside = torch.cuda.Stream(), torch.cuda.Stream()
    graphs = [torch.cuda.CUDAGraph() for _ in S.GRAPHS]
    torch.cuda.synchronize()
    for i, graph in enumerate(graphs):
        with torch.cuda.graph(graph, stream=st):
            product(i, ys[i], work)
    for r in range(6):
        for i, (x, *_) in enumerate(ops):
            x.copy_(torch.randint(-127, 128, x.shape, dtype=torch.int8, device="cuda"))
            ys[i].fill_(77.0)
        torch.cuda.synchronize()
        for i, graph in enumerate(graphs):
            graph.replay()
            product(i, eager[i], other, aside)
        torch.cuda.synchronize()
        for i, (y, e) in enumerate(zip(ys, eager)):
            assert torch.equal(y, e), (r, i)
            x, xs, w, ws, bias, _ = ops[i]
            v = (x.double() @ w.double().t().contiguous()) * xs.double()[:, None] * ws.double()
            tol = 3 * IO.U * v.abs()
            v = v + bias
            assert ((y.double() - v).abs() <= (tol + IO.U * v.abs()) * (1 + 2.0 ** -20)).all(), (r, i)
