"""Attention over the 4-bit cache where the factor of a row's scores passes float32's range and the
scores do not: they are 0, and the row is the mean of the values that it sees.  Tolerance: that of
test_gpu_attend.py."""

import numpy as np
import pytest
import torch

from oracle import cache as oc
from tests.cache_setup import Setup
from tests.test_gpu_attend import queries, within

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def tv():
    import paper_2505_12398_gb300 as tv
    from paper_2505_12398_gb300.build import build
    build()
    return tv


@pytest.mark.parametrize("scale", [1e38, -1e38])
@pytest.mark.parametrize("d,G,R", [(128, 4, 1), (64, 4, 3), (128, 4, 20), (64, 4, 50)])
def test_rows_of_zeros_under_a_large_scale(tv, d, G, R, scale):
    n = 200
    s = Setup(tv, [n], R, 1, d, 16, seed=7)
    s.np_exp[:], s.np_exp[0, 0] = 0, 40
    s.cache.exponents.copy_(torch.from_numpy(s.np_exp))
    held = s.fill(extra=R)
    q = torch.zeros(1, R, G, d, dtype=torch.bfloat16)
    got = s.cache.attend(0, q.cuda(), s.lengths, s.table, scale=scale)
    assert s.v.status() == 0
    K, V = held[0]
    mask = oc.visible(None, n, R)
    want = oc.attention(np.zeros((R, G, d)), K, V, mask, 1.0)
    A = oc.attention(np.zeros((R, G, d)), K, np.abs(V), mask, 1.0)
    within(got[0].double().cpu().numpy(), want, A, n + R, np.abs(V).max())
    # beside a row that is not finite, which alone is not a number
    q[0, R - 1, 1] = queries(1, 1, 1, d, 1)[0, 0, 0]
    q[0, R - 1, 1, 3] = float("nan")
    y = s.cache.attend(0, q.cuda(), s.lengths, s.table, scale=scale)
    assert bool(torch.isnan(y[0, R - 1, 1]).all())
    y[0, R - 1, 1] = got[0, R - 1, 1]
    assert torch.equal(y, got)
