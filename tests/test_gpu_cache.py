"""The 4-bit key/value cache: rows quantised as they are written, read back, and moved after
a verification, against the float64 restatement in oracle/cache.py.  The format has one answer for
every input, so that everything is compared exactly."""

import numpy as np
import pytest
import torch

from oracle import cache as oc
from tests.cache_setup import Setup

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def tv():
    import paper_2505_12398_gb300 as tv
    from paper_2505_12398_gb300.build import build
    build()
    return tv


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("d,P,Hk,R,lens", [
    (64, 16, 1, 1, [0]), (64, 16, 3, 7, [0, 5, 16, 31]), (128, 16, 2, 61, [3, 64, 200]),
    (128, 32, 1, 33, [1, 30]), (128, 64, 8, 12, [63, 64, 65, 0, 7]), (64, 128, 5, 130, [100, 1]),
    (128, 128, 2, 9, [119, 120, 127, 128])])
def test_rows_written_and_read_back(tv, dtype, d, P, Hk, R, lens):
    s = Setup(tv, lens, R, Hk, d, P, seed=R + d)
    k, v = s.rows(R, dtype), s.rows(R, dtype)
    s.cache.write(0, k.cuda(), v.cuda(), s.lengths, s.table)
    for kind in (torch.bfloat16, torch.float32):
        gk, gv = s.cache.read(0, s.lengths + R, s.table, R + 3, first=s.lengths, dtype=kind)
        assert gk.dtype == kind
        assert np.array_equal(gk[:, :R].double().cpu().numpy(), s.want(k, 0, 0))
        assert np.array_equal(gv[:, :R].double().cpu().numpy(), s.want(v, 0, 1))
        assert bool((gk[:, R:] == 0).all()) and bool((gv[:, R:] == 0).all())
    assert s.v.status() == 0


def test_bytes_are_the_documented_ones(tv):
    P, d, R = 32, 128, 3
    s = Setup(tv, [30], R, 2, d, P, layers=2, fill=0)
    k, v = s.rows(R), s.rows(R)
    s.cache.write(1, k.cuda(), v.cuda(), s.lengths, s.table)
    want = np.zeros(tuple(s.cache.data.shape), dtype=np.uint8)
    for i in range(R):
        page, slot = s.np_table[0, (30 + i) // P], (30 + i) % P
        for h in range(2):
            for side, x in ((0, k), (1, v)):
                oc.put_row(want[1, page, h, side], P, slot, x[0, i, h].double().numpy(),
                           int(s.np_exp[1, side, h]))
    got = s.cache.data.cpu().numpy()
    half = P * d // 2
    # (a code of 8 is -0, and either zero stands for one)
    lo, hi = got[..., :half] & 15, got[..., :half] >> 4
    codes = np.where(lo == 8, 0, lo) | np.where(hi == 8, 0, hi) << 4
    assert np.array_equal(codes, want[..., :half])
    assert np.array_equal(got[..., half:], want[..., half:])


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_ties_extremes_and_odd_values(tv, dtype):
    """Groups whose quotients are the middles between codes and between scales, zeros,
    subnormals, values past the format, infinities and a NaN."""
    R, d = 40, 64
    s = Setup(tv, [0], R, 1, d, 16)
    x = torch.zeros(1, R, 1, d, dtype=torch.float64)
    mids = torch.tensor([0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0, 6.0])
    for i in range(16):                                  # scales 8/8 .. 15/8, then odd powers
        sc = (8 + i % 8) / 8.0 * 2.0 ** (3 * (i // 8) - 4)
        x[0, i, 0, :8], x[0, i, 0, 8:16] = mids * sc, -mids * sc
        x[0, i, 0, 16:32] = x[0, i, 0, :16] * (1 + 2.0 ** -7)
        x[0, i, 0, 15], x[0, i, 0, 31] = 6 * sc, -6 * sc
        x[0, i, 0, 32:48] = x[0, i, 0, :16] * (1 - 2.0 ** -8)
        x[0, i, 0, 48] = 6 * (2 * (8 + i % 8) + 1) / 16.0   # a tie of the scale
    x[0, 16] = 1e-30
    x[0, 17, 0, 0] = 6 * 2.0 ** -10                      # half of the least scale
    x[0, 18, 0, 0] = 6 * 2.0 ** -10 * 1.0078125
    x[0, 19, 0, :16] = 2.0 ** -9 * torch.arange(16)
    x[0, 20, 0, :] = 3e38
    x[0, 21, 0, 5], x[0, 21, 0, 6] = float("inf"), 1.0
    x[0, 22, 0, 20] = -float("inf")
    x[0, 23] = 2688.0 * 8 * torch.linspace(-2, 2, d)
    x = x.to(dtype)
    if dtype == torch.float32:                           # one step beside every middle
        x[0, 24:32] = torch.nextafter(x[0, :8], torch.full_like(x[0, :8], 1e9))
        x[0, 32:40] = torch.nextafter(x[0, :8], torch.full_like(x[0, :8], -1e9))
    s.np_exp[:] = 0
    s.cache.exponents.zero_()
    s.cache.write(0, x.cuda(), x.cuda(), s.lengths, s.table)
    assert s.v.status() == 0
    gk, gv = s.cache.read(0, s.lengths + R, s.table, R, dtype="fp32")
    want = s.want(x, 0, 0)
    assert np.array_equal(gk.double().cpu().numpy(), want)
    assert np.array_equal(gv.double().cpu().numpy(), want)
    x[0, 3, 0, 7] = float("nan")
    s.cache.write(0, x.cuda(), x.cuda(), s.lengths, s.table)
    assert tv.status_names(s.v.status()) == ["NAN"]
    gk, _ = s.cache.read(0, s.lengths + R, s.table, R, dtype="fp32")
    assert np.array_equal(gk.double().cpu().numpy(), s.want(x, 0, 0))


def test_ragged_rows_and_what_lies_beside_them(tv):
    """Rows behind a request's last are not read and nothing is written for them."""
    R, lens, counts = 20, [7, 0, 33, 16], [20, 0, 3, 11]
    s = Setup(tv, lens, R, 2, 128, 16, fill=0x33)
    k, v = s.rows(R), s.rows(R)
    for b, n in enumerate(counts):
        k[b, n:], v[b, n:] = float("nan"), float("inf")
    before = s.cache.data.clone()
    rows = torch.tensor(counts, dtype=torch.int32, device="cuda")
    s.cache.write(0, k.cuda(), v.cuda(), s.lengths, s.table, rows=rows)
    gk, gv = s.cache.read(0, s.lengths + rows, s.table, R, first=s.lengths, dtype="fp32")
    for b, n in enumerate(counts):
        assert np.array_equal(gk[b, :n].double().cpu().numpy(), s.want(k, 0, 0)[b, :n])
        assert np.array_equal(gv[b, :n].double().cpu().numpy(), s.want(v, 0, 1)[b, :n])
        assert bool((gk[b, n:] == 0).all())
    # the rows before and behind hold the bytes that they had
    s2 = tv.KVCache(s.v, 1, s.cache.pages, 2, 128, page_size=16, data=before,
                    exponents=s.cache.exponents)
    n = 48
    full = torch.full_like(s.lengths, n)
    wide = torch.arange(s.cache.pages, dtype=torch.int32, device="cuda")[None, :3].expand(4, 3)
    table = torch.where(s.table[:, :3] < 0, wide, s.table[:, :3]).contiguous()
    a, _ = s.cache.read(0, full, table, n, dtype="fp32")
    b_, _ = s2.read(0, full, table, n, dtype="fp32")
    for b, (m, c) in enumerate(zip(lens, counts)):
        own = [p for p in range(n) if s.np_table[b, p // 16] >= 0]
        same = [p for p in own if not m <= p < m + c]
        assert torch.equal(a[b, same], b_[b, same])
    assert s.v.status() == 0


def test_bad_pages_and_lengths_are_reported(tv):
    R = 5
    s = Setup(tv, [10, 20, 4], R, 1, 64, 16)
    k = s.rows(R).cuda()
    before = s.cache.data.clone()
    table = s.table.clone()
    table[:, :] = s.cache.pages                          # every page is outside
    s.cache.write(0, k, k, s.lengths, table)
    assert tv.status_names(s.v.status()) == ["BAD_PAGE"]
    far = torch.full_like(s.lengths, 10 ** 6)            # positions outside the table
    s.cache.write(0, k, k, far, s.table)
    assert tv.status_names(s.v.status()) == ["BAD_PAGE"]
    top = torch.full_like(s.lengths, 2 ** 31 - 3)        # and past 32 bits
    s.cache.write(0, k, k, top, s.table)
    assert tv.status_names(s.v.status()) == ["BAD_PAGE"]
    s.cache.write(0, k, k, torch.full_like(s.lengths, -1), s.table)
    assert tv.status_names(s.v.status()) == ["BAD_LENGTH"]
    assert torch.equal(s.cache.data, before)
    gk, gv = s.cache.read(0, s.lengths, table, 30)
    assert tv.status_names(s.v.status()) == ["BAD_PAGE"]
    assert bool((gk == 0).all()) and bool((gv == 0).all())
    gk, _ = s.cache.read(0, s.lengths, s.table, 8, first=s.lengths - 50)
    assert tv.status_names(s.v.status()) == ["BAD_LENGTH"] and bool((gk == 0).all())
    s.cache.write(0, k, k, s.lengths, s.table,
                  rows=torch.tensor([R + 1, 2, -1], dtype=torch.int32, device="cuda"))
    assert tv.status_names(s.v.status()) == ["BAD_LENGTH"]
    gk, _ = s.cache.read(0, s.lengths + R, s.table, R, first=s.lengths, dtype="fp32")
    assert np.array_equal(gk[0].double().cpu().numpy(), s.want(k.cpu(), 0, 0)[0])


@pytest.mark.parametrize("layers,d,P", [(1, 64, 16), (3, 128, 32)])
def test_accepted_rows_follow_the_root(tv, layers, d, P):
    N = 40
    lens = [0, 5, 31, 64, 12, 9]
    paths = [[1, 2, 3], [3, 5, 6, 7, 20, 21, 22, 23, 24, 30, 39, 40], [], [40],
             list(range(1, 41)), [2]]
    tau = [3, 12, 0, 1, 40, -1]
    s = Setup(tv, lens, N + 1, 2, d, P, layers=layers)
    k, v = [s.rows(N + 1) for _ in range(layers)], [s.rows(N + 1) for _ in range(layers)]
    for i in range(layers):
        s.cache.write(i, k[i].cuda(), v[i].cuda(), s.lengths, s.table)
    path = torch.full((len(lens), N), -1, dtype=torch.int32)
    for b, p in enumerate(paths):
        path[b, :len(p)] = torch.tensor(p, dtype=torch.int32)
    t = torch.tensor(tau, dtype=torch.int32)
    new = s.cache.accept(path.cuda(), t.cuda(), s.lengths, s.table)
    want = [n + 1 + a if a >= 0 else n for n, a in zip(lens, tau)]
    assert new.tolist() == want and s.lengths.tolist() == lens
    for i in range(layers):
        gk, gv = s.cache.read(i, new, s.table, N + 1, first=s.lengths, dtype="fp32")
        wk, wv = s.want(k[i], i, 0), s.want(v[i], i, 1)
        for b in range(len(lens)):
            rows = oc.accept(paths[b], tau[b])
            assert np.array_equal(gk[b, :len(rows)].double().cpu().numpy(), wk[b, rows])
            assert np.array_equal(gv[b, :len(rows)].double().cpu().numpy(), wv[b, rows])
            assert bool((gk[b, len(rows):] == 0).all())
    assert s.v.status() == 0


def test_bad_paths_are_reported(tv):
    N = 6
    s = Setup(tv, [3, 3, 3, 3], N + 1)
    k = s.rows(N + 1).cuda()
    s.cache.write(0, k, k, s.lengths, s.table)
    before = s.cache.data.clone()
    path = torch.tensor([[2, 1, -1, -1, -1, -1], [3, 7, -1, -1, -1, -1], [0, 2, -1, -1, -1, -1],
                         [2, 2, 3, -1, -1, -1]], dtype=torch.int32, device="cuda")
    tau = torch.tensor([2, 2, 2, 3], dtype=torch.int32, device="cuda")
    new = s.cache.accept(path, tau, s.lengths, s.table)
    assert torch.equal(new, s.lengths) and torch.equal(before, s.cache.data)
    assert tv.status_names(s.v.status()) == ["BAD_PATH"]
    new = s.cache.accept(path, torch.full_like(tau, N + 1), s.lengths, s.table)
    assert torch.equal(new, s.lengths) and torch.equal(before, s.cache.data)
    assert tv.status_names(s.v.status()) == ["BAD_PATH"]


def test_another_stream_a_graph_and_the_form_for_one_token(tv):
    """Writes of one token and reads on a side stream, and both captured and replayed on
    new contents."""
    s = Setup(tv, [15, 16, 200], 1, 8, 128, 64)
    k, v = s.rows(1), s.rows(1)
    kd, vd = k.cuda(), v.cuda()
    st = torch.cuda.Stream()
    st.wait_stream(torch.cuda.current_stream())
    s.cache.write(0, kd, vd, s.lengths, s.table, stream=st)
    gk, gv = s.cache.read(0, s.lengths + 1, s.table, 1, first=s.lengths, dtype="fp32", stream=st)
    st.synchronize()
    assert np.array_equal(gk.double().cpu().numpy(), s.want(k, 0, 0))
    after = s.lengths + 1
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        s.cache.write(0, kd, vd, s.lengths, s.table)
        gk, gv = s.cache.read(0, after, s.table, 1, first=s.lengths, dtype="fp32")
    for _ in range(2):
        k, v = s.rows(1), s.rows(1)
        kd.copy_(k)
        vd.copy_(v)
        graph.replay()
        torch.cuda.synchronize()
        assert np.array_equal(gk.double().cpu().numpy(), s.want(k, 0, 0))
        assert np.array_equal(gv.double().cpu().numpy(), s.want(v, 0, 1))


def test_a_cache_past_32_bit_offsets(tv):
    """Pages whose bytes lie past 2^32 of the array."""
    P, d, Hk = 128, 128, 8
    pages = (1 << 32) // (Hk * 2 * P * d * 9 // 16) + 40
    v = tv.Verifier(1000, 7, 1, "bf16", path="three")
    cache = tv.KVCache(v, 1, pages, Hk, d, page_size=P)
    table = torch.tensor([[pages - 1, pages // 2 + 1]], dtype=torch.int32, device="cuda")
    lengths = torch.tensor([120], dtype=torch.int32, device="cuda")
    g = torch.Generator().manual_seed(5)
    k, w = (torch.randn(1, 16, Hk, d, generator=g).to(torch.bfloat16) for _ in range(2))
    cache.write(0, k.cuda(), w.cuda(), lengths, table)
    gk, gw = cache.read(0, lengths + 16, table, 16, first=lengths, dtype="fp32")
    assert np.array_equal(gk.double().cpu().numpy(), oc.held(k.double().numpy(), 0))
    assert np.array_equal(gw.double().cpu().numpy(), oc.held(w.double().numpy(), 0))
    assert v.status() == 0
    path = torch.tensor([[2, 4, 5, -1, -1, -1, -1]], dtype=torch.int32, device="cuda")
    tau = torch.tensor([3], dtype=torch.int32, device="cuda")
    new = cache.accept(path, tau, lengths, table)
    gk, _ = cache.read(0, new, table, 4, first=lengths, dtype="fp32")
    assert np.array_equal(gk.double().cpu().numpy(),
                          oc.held(k[:, [0, 2, 4, 5]].double().numpy(), 0))
