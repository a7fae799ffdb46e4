"""Attention over the 4-bit cache by tiles where a tile's largest scores grow with every 32 tokens
that it looks at, in some of a warp's rows: sums are scaled while the next scores are on their way,
and the other rows' results need all of those.  Reference and tolerance are those of
test_gpu_attend.py; scores stay below 330."""

import pytest
import torch

from oracle import cache as oc
from tests.cache_setup import Setup
from tests.test_gpu_attend import check, queries, tree

pytestmark = pytest.mark.gpu

STEP, PART = 128, 32         # tokens of a step, and of it the scores that come together


@pytest.fixture(scope="module")
def tv():
    import paper_2505_12398_gb300 as tv
    from paper_2505_12398_gb300.build import build
    build()
    return tv


def rising(s, R):
    """Cached tokens whose keys' first column grows by 6 (8.7 times log2(e), more than the 8 that
    leave sums as they are) from one 32 tokens to the next, in the order in which a tile looks
    at them: last step first."""
    n, B = max(s.lens), len(s.lens)
    g = torch.Generator().manual_seed(5)
    k = 0.5 * torch.randn(B, n, s.Hk, s.d, generator=g)
    pos = torch.arange(n)
    for b, length in enumerate(s.lens):
        last = (length + R - 1) // STEP
        k[b, :, :, 0] = 6.0 * ((last - pos // STEP) * 4 + pos % STEP // PART)[:, None]
    v = torch.randn(B, n, s.Hk, s.d, generator=g)
    s.np_exp[:] = 0
    s.cache.exponents.zero_()
    s.cache.write(0, k.cuda(), v.cuda(), torch.zeros_like(s.lengths), s.table, rows=s.lengths)
    return [(oc.held(k[b].double().numpy(), 0)[:m], oc.held(v[b].double().numpy(), 0)[:m])
            for b, m in enumerate(s.lens)]


def mixed_queries(B, R, H, d):
    """Of four neighbouring rows one's scores grow, one's grow by half as much, one's fall, and
    those of one stay as they are, so that all its tokens count."""
    q = 0.2 * queries(B, R, H, d, 8).float()
    q[..., 0] = torch.tensor([1.0, 0.0, -1.0, 0.5])[(torch.arange(R)[:, None]
                                                     + torch.arange(H)) % 4]
    return q.to(torch.bfloat16)


@pytest.mark.parametrize("d,G,R,lens", [
    (128, 4, 40, [1500, 1370]), (64, 4, 40, [1500, 1370]), (128, 1, 300, [900, 31]),
    (128, 4, 61, [120 * i + 7 * i % 50 for i in range(12)])])
def test_rows_whose_largest_score_grows_beside_others(tv, d, G, R, lens):
    """Tiles of 256 rows."""
    s = Setup(tv, lens, R, 1, d, 64, seed=3)
    held = rising(s, R)
    q = mixed_queries(len(lens), R, G, d)
    check(s, q, R, scale=1.0, held=held)
    if R <= 64:
        check(s, q, R, parents=[tree(R, b) for b in range(len(lens))], scale=1.0, held=held)


@pytest.mark.parametrize("d,G,R,lens", [
    (128, 4, 32, [1500, 1370]), (64, 4, 20, [1500, 1370]), (128, 1, 27, [900, 31]),
    (128, 16, 1, [1000, 5, 700]), (128, 4, 20, [120 * i + 7 * i % 50 for i in range(12)]),
    (64, 1, 61, [40 * i + 7 * i % 50 for i in range(100)])])
def test_two_sums_of_the_same_rows(tv, d, G, R, lens):
    """Up to 128 rows: both tiles hold sums of the same rows over alternate steps, scaled apart
    and then joined, each half of the columns by another tile's threads."""
    s = Setup(tv, lens, R, 1, d, 64, seed=3)
    held = rising(s, R)
    q = mixed_queries(len(lens), R, G, d)
    parents = [tree(R, b) for b in range(len(lens))]
    check(s, q, R, parents=parents, scale=1.0, held=held)
    check(s, q, R, scale=1.0, held=held)
    qd = q.cuda()
    first = s.cache.attend(0, qd, s.lengths, s.table, scale=1.0)
    for _ in range(20):
        assert torch.equal(first, s.cache.attend(0, qd, s.lengths, s.table, scale=1.0))
