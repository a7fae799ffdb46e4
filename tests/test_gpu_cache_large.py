"""Large writes to the 4-bit cache and large reads of it, whose warps take four strips of a row
each (but for writes of fp32): against the float64 restatement and against small calls, both
exactly, with ragged rows and lengths inside a run of 8 positions; and outputs at 16 bytes that
are not 32."""

import numpy as np
import pytest
import torch

from tests.cache_setup import Setup

pytestmark = pytest.mark.gpu

LENS, R, COUNTS = [3, 1001, 50, 16], 9000, [9000, 8993, 1, 4501]


@pytest.fixture(scope="module")
def tv():
    import paper_2505_12398_gb300 as tv
    from paper_2505_12398_gb300.build import build
    build()
    return tv


def ints(x):
    return torch.tensor(x, dtype=torch.int32, device="cuda")


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("d,P,Hk", [(64, 16, 1), (64, 128, 3), (128, 64, 1), (128, 32, 2)])
def test_large_calls(tv, dtype, d, P, Hk):
    s = Setup(tv, LENS, R, Hk, d, P, seed=d + Hk, fill=0x33)
    k, v = s.rows(R, dtype), s.rows(R, dtype)
    kd, vd, rows = k.cuda(), v.cuda(), ints(COUNTS)
    small = tv.KVCache(s.v, 1, s.cache.pages, Hk, d, page_size=P, data=s.cache.data.clone(),
                       exponents=s.cache.exponents)
    s.cache.write(0, kd, vd, s.lengths, s.table, rows=rows)
    piece = 100
    for at in range(0, R, piece):
        small.write(0, kd[:, at:at + piece].contiguous(), vd[:, at:at + piece].contiguous(),
                    s.lengths + at, s.table, rows=(rows - at).clamp(0, piece))
    assert torch.equal(s.cache.data, small.data)
    del small
    wk, wv = s.want(k, 0, 0), s.want(v, 0, 1)
    for kind in (torch.bfloat16, torch.float32):
        gk, gv = s.cache.read(0, s.lengths + rows, s.table, R + 3, first=s.lengths, dtype=kind)
        for b, n in enumerate(COUNTS):
            assert np.array_equal(gk[b, :n].double().cpu().numpy(), wk[b, :n])
            assert np.array_equal(gv[b, :n].double().cpu().numpy(), wv[b, :n])
            assert not bool(gk[b, n:].any()) and not bool(gv[b, n:].any())
    assert s.v.status() == 0


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("n", [21, 9000])
def test_outputs_that_are_not_at_32_bytes(tv, dtype, n):
    lens, Hk, d = [9013, 17, 0, 4000], 1, 64
    s = Setup(tv, lens, 0, Hk, d, 16, seed=4)
    s.fill()
    first = ints([5, 0, 0, 3991])
    want = s.cache.read(0, s.lengths, s.table, n, first=first, dtype=dtype)
    size, off = len(lens) * n * Hk * d, 16 // dtype.itemsize
    for which in range(2):                           # one of both outputs, so that both are
        out, around = [], []
        for i in range(2):
            at = off if i == which else 0
            x = torch.full((size + 2 * off,), 7.0, dtype=dtype, device="cuda")
            out.append(x[at:at + size].view(len(lens), n, Hk, d))
            around.append((x, at))
        assert out[which].data_ptr() % 32 == 16
        s.cache.read(0, s.lengths, s.table, n, first=first, dtype=dtype, out=tuple(out))
        for y, w, (x, at) in zip(out, want, around):
            assert torch.equal(y, w)
            assert bool((x[:at] == 7).all()) and bool((x[at + size:] == 7).all())
    assert s.v.status() == 0
