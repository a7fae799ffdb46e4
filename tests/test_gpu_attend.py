"""Attention of drafted trees, prompts and single tokens over the 4-bit cache against the
float64 restatement in oracle/cache.py, at the sizes and masks where it can go wrong.

Tolerance, per element, with A the attention over |v| under the same weights: the output is
rounded once to bf16 (2^-8 of it), every weight once to fp16 (2^-11 of itself, so of A), and
scores in float32, sums of up to 128 products of magnitude S in all, are off by up to about
2^-21 S, which the tests keep below 2^-12 (S < 500); a weight's error and its sum's both count.
Weights below fp16's normal range are rounded to multiples of 2^-24 where the largest is 2^-2 or
more times 2^8 (2^6 and up): n of them add at most n 2^-31 of the largest |v|."""

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


def within(got, want, weight_of_abs, n, top):
    tol = 2.0 ** -8 * np.abs(want) + (2.0 ** -11 + 2.0 ** -11) * weight_of_abs + \
        n * 2.0 ** -31 * top
    err = np.abs(got - want)
    assert not np.isnan(got).any()
    assert np.all(err <= tol), (float((err - tol).max()), float(err.max()), np.argwhere(err > tol)[:4])


def tree(R, seed, fan=3):
    """Random parents: node i hangs on one of a few before it."""
    rng = np.random.default_rng(seed)
    return [-1] + [int(rng.integers(max(0, (i - 1) // fan - 2), i)) for i in range(1, R)]


def check(s, q, R, parents=None, counts=None, scale=None, layer=0, out=None, held=None):
    """Writes R rows behind the cached tokens, attends, and compares every request."""
    B = len(s.lens)
    held = s.fill(layer) if held is None else held
    k, v = s.rows(R, spread=1.0), s.rows(R, spread=1.0)
    rows = None if counts is None else torch.tensor(counts, dtype=torch.int32, device="cuda")
    s.cache.write(layer, k.cuda(), v.cuda(), s.lengths, s.table, rows=rows)
    wk, wv = s.want(k, layer, 0), s.want(v, layer, 1)
    par = None if parents is None else torch.tensor(parents, dtype=torch.int32, device="cuda")
    got = s.cache.attend(layer, q.cuda(), s.lengths, s.table, parents=par, rows=rows, scale=scale,
                         out=out)
    again = s.cache.attend(layer, q.cuda(), s.lengths, s.table, parents=par, rows=rows,
                           scale=scale)
    assert torch.equal(got, again)                 # (no order that changes)
    assert s.v.status() == 0
    f = s.d ** -0.5 if scale is None else scale
    got = got.double().cpu().numpy()
    for b in range(B):
        r = R if counts is None else counts[b]
        assert not got[b, r:].any()
        if r == 0:
            continue
        K = np.concatenate([held[b][0][:s.lens[b]], wk[b, :r]])
        V = np.concatenate([held[b][1][:s.lens[b]], wv[b, :r]])
        mask = oc.visible(None if parents is None else parents[b], s.lens[b], r)
        qb = q[b, :r].double().numpy()
        want = oc.attention(qb, K, V, mask, f)
        A = oc.attention(qb, K, np.abs(V), mask, f)
        within(got[b, :r], want, A, len(K), np.abs(V).max())
    return got


def queries(B, R, H, d, seed, spread=0.0):
    g = torch.Generator().manual_seed(seed)
    q = torch.randn(B, R, H, d, generator=g)
    return (q * torch.exp2(spread * (2 * torch.rand(B, R, H, 1, generator=g) - 1))).to(
        torch.bfloat16)


LENS = [0, 1, 15, 16, 17, 127, 128, 129, 300, 1000]


@pytest.mark.parametrize("d,P", [(64, 16), (64, 128), (128, 16), (128, 32), (128, 64), (128, 128)])
@pytest.mark.parametrize("Hk,G", [(1, 1), (2, 4), (3, 5), (1, 8), (2, 16), (1, 40)])
def test_one_token(tv, d, P, Hk, G):
    s = Setup(tv, LENS, 1, Hk, d, P, seed=d + P + G)
    check(s, queries(len(LENS), 1, Hk * G, d, G), 1)


@pytest.mark.parametrize("d,P,Hk,G,R", [
    (64, 16, 2, 1, 27), (64, 64, 1, 4, 9), (128, 16, 1, 1, 8), (128, 64, 2, 2, 5),
    (128, 128, 1, 4, 61), (128, 32, 2, 3, 33), (64, 32, 1, 8, 31), (128, 16, 1, 1, 200),
    (64, 128, 1, 2, 121), (128, 64, 1, 16, 27)])
def test_trees(tv, d, P, Hk, G, R):
    """Every request has its own tree, which ends anywhere in a page and in a tile."""
    lens = [0, 1, 100, 127, 128, 390]
    s = Setup(tv, lens, R, Hk, d, P, seed=R, nodes=max(R - 1, 1))
    check(s, queries(len(lens), R, Hk * G, d, R), R, parents=[tree(R, 10 * R + b) for b in range(6)])


@pytest.mark.parametrize("d,P,Hk,G,R,counts", [
    (64, 16, 2, 1, 40, [40, 0, 1, 17, 39]), (128, 64, 1, 4, 150, [150, 149, 64, 0, 3]),
    (128, 16, 2, 2, 300, [1, 300, 129, 255, 31]), (64, 128, 1, 3, 130, [130, 100, 77, 2, 0]),
    (128, 128, 1, 7, 100, [37, 73, 100, 99, 1])])
def test_prompts_of_ragged_rows(tv, d, P, Hk, G, R, counts):
    lens = [0, 9, 128, 250, 1]
    s = Setup(tv, lens, R, Hk, d, P, seed=R + 1)
    check(s, queries(5, R, Hk * G, d, R), R, counts=counts)


def test_trees_of_ragged_rows(tv):
    """A tree cut short: its first rows, an ancestor of each among them."""
    lens, R = [33, 0, 500], 60
    s = Setup(tv, lens, R, 2, 128, 32, seed=4)
    check(s, queries(3, R, 8, 128, 3), R, parents=[tree(R, b) for b in range(3)],
          counts=[60, 13, 0])


@pytest.mark.parametrize("d,G", [(64, 1), (128, 2)])
def test_the_largest_tree_and_a_chain(tv, d, G):
    R = 1024
    s = Setup(tv, [70, 3], R, 1, d, 64, nodes=1023, seed=9)
    chain = list(range(-1, R - 1))
    check(s, queries(2, R, G, d, 1), R, parents=[chain, tree(R, 5)])


@pytest.mark.parametrize("d,G,R", [(128, 4, 1), (64, 2, 3), (128, 4, 9), (128, 8, 27)])
def test_loud_queries_and_scales(tv, d, G, R):
    """Rows of queries over many powers of two, a scale of its own, several layers, and
    scores of which few or all tokens count."""
    s = Setup(tv, [700, 5, 64], R, 2, d, 16, layers=3, seed=11)
    par = [tree(R, b) for b in range(3)]
    check(s, queries(3, R, 2 * G, d, 2, spread=4.0), R, parents=par, layer=2)
    s.np_exp[:] = 0
    s.cache.exponents.zero_()
    check(s, queries(3, R, 2 * G, d, 3), R, parents=par, scale=0.3)
    check(s, queries(3, R, 2 * G, d, 3), R, parents=par, scale=-0.05)
    check(s, queries(3, R, 2 * G, d, 3), R, parents=par, scale=0.0)


@pytest.mark.parametrize("R", [1, 20])
def test_powers_of_two_change_nothing_else(tv, R):
    """Queries times a power of two (to the ends of bf16's range) and the scale over it give
    the same bits; so do exponents."""
    s = Setup(tv, [333], R, 1, 128, 16, seed=2)
    s.np_exp[:] = 0
    s.cache.exponents.zero_()
    q = queries(1, R, 4, 128, 5)
    base = check(s, q, R)
    for e in (-100, -20, 30, 100):
        y = s.cache.attend(0, (q.float() * 2.0 ** e).to(torch.bfloat16).cuda(), s.lengths, s.table,
                           scale=128 ** -0.5 * 2.0 ** -e)
        assert np.array_equal(y.double().cpu().numpy(), base)
    s.cache.exponents[0, 0, 0], s.cache.exponents[0, 1, 0] = 7, -9
    y = s.cache.attend(0, q.cuda(), s.lengths, s.table, scale=128 ** -0.5 * 2.0 ** -7)
    assert np.array_equal(y.double().cpu().numpy() * 512, base)


@pytest.mark.parametrize("R", [1, 5, 50])
def test_rising_scores(tv, R):
    """The largest score keeps moving up along the tokens (and down), by far more than the
    slack that leaves a sum as it is."""
    n, d = 1500, 128
    s = Setup(tv, [n, n], R, 1, d, 64, seed=3)
    s.np_exp[:] = 0
    s.cache.exponents.zero_()
    g = torch.Generator().manual_seed(7)
    k = torch.zeros(2, n, 1, d)
    k[0, :, 0, 0] = torch.linspace(0, 300, n)
    k[1, :, 0, 0] = torch.linspace(300, 0, n)
    k[..., 1:] = 0.5 * torch.randn(2, n, 1, d - 1, generator=g)
    v = torch.randn(2, n, 1, d, generator=g)
    zero = torch.zeros_like(s.lengths)
    s.cache.write(0, k.cuda(), v.cuda(), zero, s.table)
    held = [(oc.held(k[b].double().numpy(), 0), oc.held(v[b].double().numpy(), 0))
            for b in range(2)]
    q = queries(2, R, 4, d, 8)
    q[..., 0] = 1.0
    check(s, q, R, scale=1.0, held=held)


@pytest.mark.parametrize("R", [1, 40])
def test_rows_that_are_not_finite(tv, R):
    """An infinity or a NaN in a row of queries makes that row NaN and no other."""
    s = Setup(tv, [100, 7], R, 1, 64, 16, seed=6)
    q = queries(2, R, 4, 64, 1)
    clean = check(s, q, R)
    for bad in (float("inf"), -float("inf"), float("nan")):
        q2 = q.clone()
        q2[1, R - 1, 2, 5] = bad
        y = s.cache.attend(0, q2.cuda(), s.lengths, s.table).double().cpu().numpy()
        assert np.isnan(y[1, R - 1, 2]).all()
        y[1, R - 1, 2] = clean[1, R - 1, 2]
        assert np.array_equal(y, clean)


@pytest.mark.parametrize("R", [1, 30])
def test_tokens_without_a_page_are_left_out(tv, R):
    P, lens = 16, [100, 40]
    s = Setup(tv, lens, R, 1, 128, P, seed=8)
    q = queries(2, R, 4, 128, 2)
    held = s.fill(extra=R)
    par = [tree(R, 3), tree(R, 4)]
    parents = torch.tensor(par, dtype=torch.int32, device="cuda")
    table = s.table.clone()
    table[0, 2], table[0, 4], table[1, 0] = -1, s.cache.pages, 2 ** 31 - 1
    gone = {0: [2, 4], 1: [0]}
    got = s.cache.attend(0, q.cuda(), s.lengths, table, parents=parents)
    assert tv.status_names(s.v.status()) == ["BAD_PAGE"]
    for b in range(2):
        mask = oc.visible(par[b], lens[b], R)
        for p in gone[b]:
            mask[:, P * p:P * p + P] = False
        K, V = held[b]
        want = oc.attention(q[b].double().numpy(), K, V, mask, 128 ** -0.5)
        A = oc.attention(q[b].double().numpy(), K, np.abs(V), mask, 128 ** -0.5)
        within(got[b].double().cpu().numpy(), want, A, len(K), np.abs(V).max())
    # none at all, and a table too short for the length
    got = s.cache.attend(0, q.cuda(), s.lengths, torch.full_like(table, -1), parents=parents)
    assert tv.status_names(s.v.status()) == ["BAD_PAGE"] and not bool(got.any())
    short = s.table[:, :2].contiguous()
    got = s.cache.attend(0, q.cuda(), s.lengths, short, parents=parents)
    assert tv.status_names(s.v.status()) == ["BAD_PAGE"]
    for b in range(2):
        K, V = held[b][0][:2 * P], held[b][1][:2 * P]
        mask = np.ones((R, 2 * P), dtype=bool)
        want = oc.attention(q[b].double().numpy(), K, V, mask, 128 ** -0.5)
        A = oc.attention(q[b].double().numpy(), K, np.abs(V), mask, 128 ** -0.5)
        within(got[b].double().cpu().numpy(), want, A, len(K), np.abs(V).max())
    got = s.cache.attend(0, q.cuda(), torch.full_like(s.lengths, 2 ** 31 - 5), short)
    assert tv.status_names(s.v.status()) == ["BAD_PAGE"]


def test_bad_trees_and_lengths_are_reported(tv):
    R = 4
    s = Setup(tv, [20, 20, 20], R, 1, 64, 16, seed=8)
    q = queries(3, R, 2, 64, 2)
    held = s.fill(extra=R)
    par = torch.tensor([[-1, 0, 5, 1], [-1, 0, 0, 1], [0, 0, -1, 1]], dtype=torch.int32)
    got = s.cache.attend(0, q.cuda(), s.lengths, s.table, parents=par.cuda())
    assert tv.status_names(s.v.status()) == ["BAD_TREE"]
    sees = {0: [[0], [0, 1], [2], [0, 1, 3]], 1: [[0], [0, 1], [0, 2], [0, 1, 3]],
            2: [[0], [0, 1], [2], [0, 1, 3]]}
    for b in range(3):
        mask = np.zeros((R, 20 + R), dtype=bool)
        mask[:, :20] = True
        for i in range(R):
            mask[i, [20 + j for j in sees[b][i]]] = True
        K, V = held[b]
        want = oc.attention(q[b].double().numpy(), K, V, mask, 64 ** -0.5)
        A = oc.attention(q[b].double().numpy(), K, np.abs(V), mask, 64 ** -0.5)
        within(got[b].double().cpu().numpy(), want, A, len(K), np.abs(V).max())
    lengths = s.lengths.clone()
    lengths[1] = -3
    rows = torch.tensor([R, R, R + 2], dtype=torch.int32, device="cuda")
    good = s.cache.attend(0, q.cuda(), s.lengths, s.table)
    bad = s.cache.attend(0, q.cuda(), lengths, s.table, rows=rows)
    assert tv.status_names(s.v.status()) == ["BAD_LENGTH"]
    assert not bool(bad[1].any()) and torch.equal(bad[[0, 2]], good[[0, 2]])


def test_requests_that_share_pages(tv):
    """A prefix in pages of two requests, each with its own pages behind it."""
    s = Setup(tv, [64, 64], 20, 2, 128, 16, seed=12)
    held = s.fill()
    s.table[1, :4] = s.table[0, :4]
    held[1] = held[0]
    check(s, queries(2, 20, 8, 128, 4), 20, parents=[tree(20, 1), tree(20, 2)], held=held)


def _gpu_reference(cache, q, lengths, table, mask_of, scale):
    """Attention in float64 on the GPU from what the cache reads back."""
    B, R, H, d = q.shape
    out, A = [], []
    n = int(lengths.max()) + R
    for b in range(B):
        t = int(lengths[b]) + R
        one = torch.full((1,), t, dtype=torch.int32, device="cuda")
        k, v = cache.read(0, one, table[b:b + 1].contiguous(), t, dtype="fp32")
        g = H // cache.kv_heads
        res = torch.empty(R, H, d, dtype=torch.float64, device="cuda")
        ab = torch.empty_like(res)
        for h in range(H):
            s = q[b, :, h].double() @ k[0, :, h // g].double().T * scale
            s = s.masked_fill(~mask_of(b, t - R), -float("inf"))
            p = torch.softmax(s, dim=1)
            res[:, h] = p @ v[0, :, h // g].double()
            ab[:, h] = p @ v[0, :, h // g].double().abs()
        out.append(res)
        A.append(ab)
    return torch.stack(out), torch.stack(A), n


@pytest.mark.parametrize("lens,Hk,G,R,d,P", [
    ([50000], 2, 4, 1, 128, 64), ([131000, 3], 1, 4, 61, 128, 64), ([20001], 1, 1, 27, 64, 16),
    ([9000, 100, 30, 1, 4000, 0, 77, 20000], 4, 2, 9, 128, 128),
    ([700 * (i % 7) + i for i in range(100)], 2, 8, 1, 128, 32),
    ([300 * (i % 5) + i for i in range(60)], 2, 4, 61, 128, 64)])
def test_long_and_many(tv, lens, Hk, G, R, d, P):
    """Items that span many CTAs, CTAs that span many items."""
    s = Setup(tv, lens, R, Hk, d, P, seed=1, nodes=max(R - 1, 1))
    g = torch.Generator(device="cuda").manual_seed(3)
    zero = torch.zeros_like(s.lengths)
    rows = s.lengths + R
    for c in range(0, max(lens) + R, 8192):        # (in pieces: the rows take memory)
        m = min(8192, max(lens) + R - c)
        k = torch.randn(len(lens), m, Hk, d, generator=g, device="cuda").to(torch.bfloat16)
        s.cache.write(0, k, -k.flip(1), zero + c, s.table,
                      rows=(rows - c).clamp(0, m).to(torch.int32))
    parents = tree(R, 7)
    m = torch.from_numpy(oc.visible(parents, 0, R)).cuda()
    par = torch.tensor([parents] * len(lens), dtype=torch.int32, device="cuda")
    q = queries(len(lens), R, Hk * G, d, 6).cuda()
    got = s.cache.attend(0, q, s.lengths, s.table, parents=par)
    assert torch.equal(got, s.cache.attend(0, q, s.lengths, s.table, parents=par))
    assert s.v.status() == 0

    def mask_of(b, n):
        return torch.cat([torch.ones(R, n, dtype=torch.bool, device="cuda"), m], dim=1)

    want, A, n = _gpu_reference(s.cache, q, s.lengths, s.table, mask_of, d ** -0.5)
    want, A = want.cpu().numpy(), A.cpu().numpy()
    within(got.double().cpu().numpy(), want, A, n, 8.0)


def test_a_graph_replayed_on_new_lengths(tv):
    """Captured once, replayed on other queries, lengths and rows; eager calls of other
    shapes on the handle in between."""
    lens, R = [200, 3000, 17], 12
    s = Setup(tv, lens, R, 2, 128, 32, seed=5)
    s.fill(extra=R)
    q = queries(3, R, 8, 128, 1).cuda()
    par = torch.tensor([tree(R, b) for b in range(3)], dtype=torch.int32, device="cuda")
    lengths = s.lengths.clone()
    s.cache.attend(0, q, lengths, s.table, parents=par)          # (the first call allocates)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = s.cache.attend(0, q, lengths, s.table, parents=par)
        one = s.cache.attend(0, q[:, :1].contiguous(), lengths, s.table)
    for seed, new in ((2, lens), (3, [0, 700, 10]), (4, [199, 1, 17])):
        q.copy_(queries(3, R, 8, 128, seed))
        lengths.copy_(torch.tensor(new, dtype=torch.int32))
        graph.replay()
        torch.cuda.synchronize()
        want = s.cache.attend(0, q, lengths, s.table, parents=par)
        assert torch.equal(out, want)
        first = s.cache.attend(0, q[:, :1].contiguous(), lengths, s.table)
        assert torch.equal(one, first)
    assert s.v.status() == 0


def test_the_first_call_may_not_be_captured(tv):
    s = Setup(tv, [20], 1, 1, 64, 16)
    s.fill(extra=1)
    q = queries(1, 1, 2, 64, 1).cuda()
    x = torch.zeros(4, device="cuda")
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        x += 1
        with pytest.raises(tv.LibraryError) as e:
            s.cache.attend(0, q, s.lengths, s.table)
    assert e.value.code == -1
    graph.replay()
    check(s, q.cpu(), 1)


def test_streams_and_given_outputs(tv):
    s = Setup(tv, [90, 400], 6, 2, 64, 16, seed=5)
    s.fill(extra=6)
    q = queries(2, 6, 4, 64, 1).cuda()
    want = s.cache.attend(0, q, s.lengths, s.table)
    st = torch.cuda.Stream()
    st.wait_stream(torch.cuda.current_stream())
    got = s.cache.attend(0, q, s.lengths, s.table, stream=st)
    out = torch.full_like(q, 5.0)
    same = s.cache.attend(0, q, s.lengths, s.table, out=out, stream=st)
    st.synchronize()
    assert same is out and torch.equal(got, want) and torch.equal(out, want)


def test_refusals(tv):
    s = Setup(tv, [20, 20], 8, 2, 64, 16, nodes=7)
    c, n, t = s.cache, s.lengths, s.table
    q = queries(2, 8, 4, 64, 1).cuda()
    par = torch.tensor([tree(8, b) for b in range(2)], dtype=torch.int32, device="cuda")
    for code, call in (
            (-1, lambda: c.attend(1, q, n, t)), (-1, lambda: c.attend(-1, q, n, t)),
            (-1, lambda: c.attend(0, q[:, :, :3].contiguous(), n, t)),
            (-1, lambda: c.attend(0, q, n, t, scale=float("nan"))),
            (-1, lambda: c.attend(0, q, n, t, out=q)),
            (-1, lambda: c.read(2, n, t, 4)),
            (-1, lambda: c.write(3, q[:, :, :2].contiguous(), q[:, :, :2].contiguous(), n, t)),
            (-1, lambda: c.accept(par[:, 1:].contiguous(), n, n, t, out=n)),
            (-4, lambda: c.attend(0, queries(2, 9, 4, 64, 1).cuda(), n, t,
                                  parents=torch.zeros(2, 9, dtype=torch.int32, device="cuda"))),
            (-4, lambda: c.attend(0, queries(3, 1, 4, 64, 1).cuda(),
                                  torch.zeros(3, dtype=torch.int32, device="cuda"),
                                  torch.zeros(3, 1, dtype=torch.int32, device="cuda"))),
            (-4, lambda: c.accept(torch.zeros(2, 8, dtype=torch.int32, device="cuda"), n, n, t))):
        with pytest.raises(tv.LibraryError) as e:
            call()
        assert e.value.code == code
    for call in (lambda: c.attend(0, q.float(), n, t), lambda: c.attend(0, q[..., :32], n, t),
                 lambda: c.attend(0, q[:, ::2], n, t),
                 lambda: c.attend(0, q, n, t, parents=par[:, :4].contiguous()),
                 lambda: c.attend(0, q, n, t, rows=n[:1]),
                 lambda: c.attend(0, q, n, t, out=torch.empty_like(q, dtype=torch.float32))):
        with pytest.raises(ValueError):
            call()
    assert s.v.status() == 0
    empty = c.attend(0, q[:, :0].contiguous(), n, t)
    assert tuple(empty.shape) == (2, 0, 4, 64)


def test_decoding_cycles(tv):
    """A tree's rows written, attended and verified, the accepted rows moved, over some
    cycles and two layers: what the cache holds is the text's rows in order, and each
    cycle's attention is that over the text and the path."""
    B, R, Hk, G, d, P, V = 3, 9, 2, 2, 64, 16, 96
    s = Setup(tv, [5, 16, 0], 80, Hk, d, P, layers=2, nodes=R - 1, seed=21)
    v = tv.Verifier(V, R - 1, B, "fp32")
    texts = [s.fill(0), s.fill(1)]
    texts = [[(list(k), list(w)) for k, w in layer] for layer in texts]
    parents = [-1, 0, 0, 1, 1, 2, 3, 3, 6]
    par = torch.tensor([parents] * B, dtype=torch.int32, device="cuda")
    g = torch.Generator(device="cuda").manual_seed(2)
    lengths = s.lengths
    moved = 0
    for cycle in range(6):
        k = [s.rows(R, spread=1.0) for _ in range(2)]
        w = [s.rows(R, spread=1.0) for _ in range(2)]
        q = queries(B, R, Hk * G, d, cycle)
        n = lengths.tolist()
        for layer in range(2):
            s.cache.write(layer, k[layer].cuda(), w[layer].cuda(), lengths, s.table)
            got = s.cache.attend(layer, q.cuda(), lengths, s.table, parents=par)
            wk, wv = s.want(k[layer], layer, 0), s.want(w[layer], layer, 1)
            for b in range(B):
                tk, tw = texts[layer][b]
                assert len(tk) == n[b]
                K = np.concatenate([np.array(tk).reshape(-1, Hk, d), wk[b]])
                W = np.concatenate([np.array(tw).reshape(-1, Hk, d), wv[b]])
                mask = oc.visible(parents, n[b], R)
                want = oc.attention(q[b].double().numpy(), K, W, mask, d ** -0.5)
                A = oc.attention(q[b].double().numpy(), K, np.abs(W), mask, d ** -0.5)
                within(got[b].double().cpu().numpy(), want, A, len(K), np.abs(W).max())
        # a verification of this tree's shape with a draft near the target
        logits = torch.randn(B, R, V, generator=g, device="cuda")
        drafts = torch.softmax(logits + 0.3 * torch.randn(B, R, V, generator=g, device="cuda"), -1)
        tokens = v.draft_children(par, drafts, torch.rand(B, R, generator=g, device="cuda"))
        path, tau, bonus = v.verify(par, tokens, logits, drafts, 1.0,
                                    torch.rand(B, R + 1, generator=g, device="cuda"))
        lengths = s.cache.accept(path, tau, lengths, s.table)
        for b in range(B):
            order = oc.accept(path[b].tolist(), int(tau[b]))
            moved += sum(i != j for i, j in enumerate(order))
            for layer in range(2):
                wk, wv = s.want(k[layer], layer, 0), s.want(w[layer], layer, 1)
                texts[layer][b][0].extend(wk[b, order])
                texts[layer][b][1].extend(wv[b, order])
    assert moved > 0 and s.v.status() == 0 and v.status() & ~16 == 0
    for layer in range(2):
        gk, gv = s.cache.read(layer, lengths, s.table, int(lengths.max()), dtype="fp32")
        for b in range(B):
            m = int(lengths[b])
            assert np.array_equal(gk[b, :m].double().cpu().numpy(), np.array(texts[layer][b][0]))
            assert np.array_equal(gv[b, :m].double().cpu().numpy(), np.array(texts[layer][b][1]))
