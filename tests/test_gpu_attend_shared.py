"""What calls of the attention over the 4-bit cache share: a handle's scratch between two captured
graphs, a GPU between two handles on two streams, and an array past 32-bit offsets.  The
tolerance is that of test_gpu_attend.py."""

import numpy as np
import pytest
import torch

from oracle import cache as oc
from tests.cache_setup import Setup
from tests.test_gpu_attend import queries, tree, within

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def tv():
    import paper_2505_12398_gb300 as tv
    from paper_2505_12398_gb300.build import build
    build()
    return tv


def _parents(R, B):
    return torch.tensor([tree(R, b) for b in range(B)], dtype=torch.int32, device="cuda")


@pytest.mark.parametrize("d,R", [(128, 1), (64, 12), (128, 40)])
def test_two_graphs_of_one_handle(tv, d, R):
    """A cycle's calls captured twice, on other queries, lengths and rows; the graphs are
    replayed in turn, eager calls between them, and give what eager calls give."""
    lens = [40, 2000, 0]
    s = Setup(tv, lens, 2 * R + 2, 2, d, 32, seed=R, nodes=max(R, 2))
    s.fill(extra=2 * R + 2)
    start = s.cache.data.clone()
    q = queries(3, R, 8, d, 1).cuda()
    s.cache.attend(0, q, s.lengths, s.table)                     # (the first call allocates)
    calls = []
    for i in range(2):
        k, v = s.rows(R, spread=1.0).cuda(), s.rows(R, spread=1.0).cuda()
        qi = queries(3, R, 8, d, 5 + i).cuda()
        n = (s.lengths - 7 * i).clamp(min=0)
        par = _parents(R, 3) if R > 1 else None
        path = torch.full((3, max(R - 1, 1)), -1, dtype=torch.int32, device="cuda")
        path[:, 0] = R - 1
        tau = torch.tensor([min(R - 1, 1), 0, -1], dtype=torch.int32, device="cuda")

        def cycle(k=k, v=v, qi=qi, n=n, par=par, path=path, tau=tau):
            s.cache.write(0, k, v, n, s.table)
            y = s.cache.attend(0, qi, n, s.table, parents=par)
            new = s.cache.accept(path, tau, n, s.table)
            return (y, new) + s.cache.read(0, new, s.table, R + 1, first=n)
        calls.append(cycle)
    want = []
    for c in calls + calls:
        want.append([x.clone() for x in c()])
    s.cache.data.copy_(start)
    graphs = []
    for c in calls:
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            out = c()
        graphs.append((g, out))
    s.cache.data.copy_(start)
    for i in range(4):
        g, out = graphs[i % 2]
        g.replay()
        s.cache.attend(0, q, s.lengths, s.table)
        torch.cuda.synchronize()
        for x, y in zip(out, want[i]):
            assert torch.equal(x, y)
    assert s.v.status() == 0


@pytest.mark.parametrize("d", [64, 128])
def test_two_handles_on_two_streams(tv, d):
    """Calls of two handles at once, of few rows and of many."""
    a = Setup(tv, [3000, 500], 61, 2, d, 64, seed=1)
    b = Setup(tv, [100, 4000], 61, 2, d, 64, seed=2)
    cases = []
    for s in (a, b):
        s.fill(extra=61)
        for R in (1, 61):
            q = queries(2, R, 8, d, R).cuda()
            par = _parents(R, 2)
            cases.append((s, q, par, s.cache.attend(0, q, s.lengths, s.table, parents=par)))
    torch.cuda.synchronize()
    streams = {a: torch.cuda.Stream(), b: torch.cuda.Stream()}
    got = []
    for _ in range(20):
        for s, q, par, want in cases:
            got.append((s.cache.attend(0, q, s.lengths, s.table, parents=par, stream=streams[s]),
                        want))
    torch.cuda.synchronize()
    for x, y in got:
        assert torch.equal(x, y)
    assert a.v.status() == 0 and b.v.status() == 0


@pytest.mark.parametrize("R", [1, 30])
def test_pages_past_32_bit_offsets(tv, R):
    P, d, Hk = 128, 128, 8
    pages = (1 << 32) // (Hk * 2 * P * d * 9 // 16) + 40
    v = tv.Verifier(1000, 40, 1, "bf16", path="three")
    cache = tv.KVCache(v, 1, pages, Hk, d, page_size=P)
    table = torch.tensor([[pages - 1, 3, pages - 30]], dtype=torch.int32, device="cuda")
    n = 300
    zero = torch.zeros(1, dtype=torch.int32, device="cuda")
    g = torch.Generator().manual_seed(5)
    k, w = (torch.randn(1, n + R, Hk, d, generator=g).to(torch.bfloat16) for _ in range(2))
    cache.write(0, k.cuda(), w.cuda(), zero, table)
    q = queries(1, R, Hk, d, 2)
    got = cache.attend(0, q.cuda(), zero + n, table).double().cpu().numpy()
    K, W = oc.held(k[0].double().numpy(), 0), oc.held(w[0].double().numpy(), 0)
    mask = oc.visible(None, n, R)
    want = oc.attention(q[0].double().numpy(), K, W, mask, d ** -0.5)
    A = oc.attention(q[0].double().numpy(), K, np.abs(W), mask, d ** -0.5)
    within(got[0], want, A, n + R, np.abs(W).max())
    assert v.status() == 0


def test_scales_that_are_no_float32_times_log2e(tv):
    s = Setup(tv, [20], 1, 1, 64, 16)
    s.fill(extra=1)
    q = queries(1, 1, 2, 64, 1).cuda()
    for scale in (3e38, -3e38, float("inf")):
        with pytest.raises(tv.LibraryError) as e:
            s.cache.attend(0, q, s.lengths, s.table, scale=scale)
        assert e.value.code == -1
    assert s.v.status() == 0


def test_more_rows_than_an_index_has_are_refused(tv):
    """By the host, from sizes alone."""
    s = Setup(tv, [20], 1, 1, 64, 16)
    lib, z = s.v.lib, None
    at = s.cache.data.data_ptr()
    n, t = s.lengths.data_ptr(), s.table.data_ptr()
    pages = s.table.shape[1]
    for rows in (2 ** 31 - 1, 2 ** 31 - 10):
        assert lib.tv_cache_read(s.v.handle, s.cache.ref, 0, 1, rows, 0, n, t, pages, z, at, at,
                                 z) == -1
        assert lib.tv_cache_write(s.v.handle, s.cache.ref, 0, 1, rows, 0, at, at, n, t, pages, z,
                                  z) == -1
    assert s.v.status() == 0
