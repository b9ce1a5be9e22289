"""The cuts of products in 8-bit integers (CPU): the workspace holds the parts of every
product that it has to serve, and is no larger than tiles that are cut need; the GPU tests run every form that
a product may be cut into."""
import numpy as np

from paper_2504_03651_amd import int8
from tests import int8_sizes as S
from tests.int8_cuts import cuts
from tests.test_gpu_int8 import SIZES


def _sizes(n, seed):
    g = np.random.default_rng(seed)
    log = lambda lo, hi: np.exp(g.uniform(np.log(lo), np.log(hi), n)).astype(np.int64)   # noqa: E731
    T, N, K, f = log(1, 5000), log(1, 40000), 16 * log(1, 1024), g.integers(0, 2, n)
    return [tuple(map(int, s)) for s in zip(T, N, K, f)]


def test_the_workspace_holds_the_parts_of_every_smaller_batch():
    sizes = _sizes(4000, 1)
    g = np.random.default_rng(2)
    for (T, N, K, f), c in zip(sizes, cuts(sizes)):
        assert c[3] <= c[4] == int8.gemm_workspace_bytes(T, N, K) <= 256 << 20
        assert (c[1] == 1) == (c[3] == 0)
    sizes = sizes[:1000]
    fewer = [(int(g.integers(1, T + 1)), N, K, f) for T, N, K, f in sizes]
    for one, all_ in zip(cuts(fewer), cuts(sizes)):
        assert one[3] <= one[4] <= all_[4]


def test_tiles_that_are_never_cut_ask_for_no_workspace():
    """Those of 256 x 192: the most is that of 256 x 128, in 2,048 tiles."""
    for N, K in [(28672, 4096), (20000, 8192), (14000, 2048)]:
        assert int8.gemm_workspace_bytes(10 ** 6, N, K) == 2048 // -(-N // 256) * 128 * N * 4 < 256 << 20


def test_every_cut_has_a_case():
    """Forms, variants and ranges of 300,000 sizes."""
    cases = [(t, n, k, f) for t, n, k in SIZES for f in (0, 1)] + S.FORMS
    have = {(s[3], *c[:3]) for s, c in zip(cases, cuts(cases))}
    seen = {}
    sizes = _sizes(300000, 3)
    for s, c in zip(sizes, cuts(sizes)):
        seen.setdefault((s[3], *c[:3]), s)
    assert len(seen) >= 120
    assert {k: s for k, s in seen.items() if k not in have} == {}


def test_products_of_shared_and_concurrent_workspaces_use_them():
    for f in (0, 1):
        for sizes in (S.STREAMS, S.GRAPHS):
            assert all(c[1] > 1 for c in cuts([(*s, f) for s in sizes]))
        for n, k in S.WEIGHTS:
            assert len({c[1] for c in cuts([(t, n, k, f) for t in S.BATCHES])}) >= 4
