"""Requests of a batch for which there is nothing to write to the 4-bit cache or to read from it:
they have no pages, their lengths are whatever an idle slot holds, and nothing is reported."""

import numpy as np
import pytest
import torch

from tests.cache_setup import Setup

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def tv():
    import paper_2505_12398_gb300 as tv
    from paper_2505_12398_gb300.build import build
    build()
    return tv


def ints(x):
    return torch.tensor(x, dtype=torch.int32, device="cuda")


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("R", [5, 3000])
def test_no_rows_to_write(tv, dtype, R):
    """Row counts of 0 behind lengths that do and do not begin a run of 8 positions."""
    lens = [13, 0, 8, 127, 2 ** 31 - 3, 20, 1, 15]
    s = Setup(tv, [20] * len(lens), R, 8, 64, 16)
    k = s.rows(R, dtype).cuda()
    before = s.cache.data.clone()
    gone = torch.full_like(s.table, -1)
    s.cache.write(0, k, k, ints(lens), gone, rows=ints([0] * len(lens)))
    assert s.v.status() == 0
    assert torch.equal(s.cache.data, before)
    rows = ints([0, 0, 0, 0, 0, 2, 0, 0])            # (one request has some, and no pages)
    s.cache.write(0, k, k, ints(lens), gone, rows=rows)
    assert tv.status_names(s.v.status()) == ["BAD_PAGE"]
    assert torch.equal(s.cache.data, before)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("n", [4, 3000])
def test_nothing_to_read(tv, dtype, n):
    """First positions at and behind the lengths, whose pages there are none of."""
    first = [13, 100, 8, 2 ** 31 - 3, 5, 0, 15, 13]
    lens = [13, 10, 8, 2 ** 31 - 4, 0, 0, 1, 20]
    s = Setup(tv, [20] * len(lens), 1, 8, 64, 16)
    gone = torch.full_like(s.table, -1)
    gone[7] = s.table[7]                             # (the last one has rows and pages)
    k = s.rows(7, dtype)
    s.cache.write(0, k.cuda(), k.cuda(), ints(first), s.table, rows=ints([0] * 7 + [7]))
    assert s.v.status() == 0
    gk, gv = s.cache.read(0, ints(lens), gone, n, first=ints(first), dtype=dtype)
    assert s.v.status() == 0
    assert not bool(gk[:7].any()) and not bool(gv[:7].any())
    m = min(n, 7)
    assert np.array_equal(gk[7, :m].double().cpu().numpy(), s.want(k, 0, 0)[7, :m])
    assert np.array_equal(gv[7, :m].double().cpu().numpy(), s.want(k, 0, 1)[7, :m])
    assert not bool(gk[7, m:].any()) and not bool(gv[7, m:].any())


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_the_lowest_lengths_are_empty(tv, dtype):
    """Negative lengths, so low that first positions taken from them pass 32 bits."""
    s = Setup(tv, [20] * 4, 0, 2, 64, 16)
    s.fill()
    first = ints([1, 5, 19, 2 ** 31 - 1])
    for low in (-2 ** 31, -2 ** 31 + 3, -1):
        gk, gv = s.cache.read(0, torch.full_like(first, low), s.table, 12, first=first,
                              dtype=dtype)
        assert tv.status_names(s.v.status()) == ["BAD_LENGTH"]
        assert not bool(gk.any()) and not bool(gv.any())
