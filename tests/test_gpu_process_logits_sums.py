"""Row sums of tv_process_logits where they are kept in more than one form: maxima on both
sides of 2^20 T / log2(e), beyond which a row is summed from differences, NaN (whose block
is summed that way too) beside large maxima, and the smallest temperatures.

Tolerance: an exponential is within 2e-7, and a thread's sum passes at most two factors of
that accuracy at each of its steps (five here at most) on its way between the forms; with
2e-6 for the rest of the sum that is 4e-6."""

import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu

LOG2E = 1.4426950408889634


@pytest.fixture(scope="module")
def tv():
    import paper_2505_12398_gb300 as tv
    from paper_2505_12398_gb300.build import build
    build()
    return tv


def _stats(tv, logits, T):
    rows, V = logits.shape
    v = tv.Verifier(V, 0, rows, "bf16" if logits.dtype == torch.bfloat16 else "fp32", path="three")
    z = torch.zeros(rows, 1, dtype=torch.int32, device="cuda")
    res, st = v.process_logits(None, z - 1, z, logits.view(rows, 1, V), T)
    assert v.status() == 0
    assert torch.equal(torch.nan_to_num(res.view(rows, V), 7.0), torch.nan_to_num(logits, 7.0))
    v.close()
    return st.view(rows, 2).double()


def _check(tv, logits, T):
    st = _stats(tv, logits, T)
    T = float(np.float32(T))                 # (as the library receives it)
    for lo in range(0, logits.shape[0], 100):
        l = logits[lo:lo + 100].double()
        nan = torch.isnan(l)
        m = torch.where(nan, torch.full_like(l, -float("inf")), l).amax(dim=1)
        s = torch.where(nan, torch.zeros_like(l), torch.exp((l - m[:, None]) / T)).sum(dim=1)
        got = st[lo:lo + 100]
        assert torch.equal(got[:, 0], m)
        assert float(((got[:, 1] - s).abs() / s).max()) <= 4e-6


def _offsets(rows, V, g, spread, run):
    """A level of its own for every ``run`` tokens."""
    n = (V + run - 1) // run
    o = (torch.rand(rows, n, generator=g, device="cuda") * 2 - 1) * spread
    return o.repeat_interleave(run, 1)[:, :V]


# 700 rows: one CTA a row, several steps a thread; 3: a cluster a row; narrow ones: 128 threads
@pytest.mark.parametrize("rows,V", [(700, 33000), (700, 33003), (3, 33003), (40000, 1003)])
@pytest.mark.parametrize("sign", [1.0, -1.0])
def test_maxima_on_both_sides(tv, rows, V, sign):
    """fp32 values within a few T of 2^20 T / log2(e): weights of blocks that are summed in
    either form matter to the same row."""
    T = 0.05
    far = 2.0 ** 20 * T / LOG2E
    g = torch.Generator(device="cuda").manual_seed(rows + V)
    l = _offsets(rows, V, g, 0.3, 8) + _offsets(rows, V, g, 0.2, 4099)
    l = (l + sign * far).float()
    # (those rows have blocks on either side)
    assert bool(((l.abs() < far).any(dim=1) & (l.abs() > far).any(dim=1)).all())
    _check(tv, l, T)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32], ids=["bf16", "fp32"])
@pytest.mark.parametrize("rows,V", [(700, 33000), (700, 33003), (3, 33003), (40000, 1003)])
@pytest.mark.parametrize("level", [30000.0, -30000.0, 127.0, 90000.0])
def test_nan_beside_large_maxima(tv, rows, V, level, dtype):
    """One NaN in some blocks (the first or the last ones of a thread, or in between)."""
    T = 0.05
    g = torch.Generator(device="cuda").manual_seed(rows + V + int(level))
    l = torch.full((rows, V), level, device="cuda")
    if dtype == torch.float32:
        l += _offsets(rows, V, g, 0.2, 8)
    else:                                    # (a bf16 step there is many T)
        l -= 512.0 * (torch.rand(rows, V, generator=g, device="cuda") < 0.5)
    l = l.to(dtype)
    blocks = torch.rand(rows, (V + 2047) // 2048, generator=g, device="cuda") < 0.5
    where = blocks.repeat_interleave(2048, 1)[:, :V] & \
        (torch.rand(rows, V, generator=g, device="cuda") < 0.02)
    l[where] = float("nan")
    _check(tv, l, T)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32], ids=["bf16", "fp32"])
@pytest.mark.parametrize("V", [1000, 1003, 33003])
@pytest.mark.parametrize("T", [5e-39, 1e-38, 1e-30, 1e30, 3e38])
def test_extreme_temperatures(tv, V, T, dtype):
    """Logits a whole number apart: at the smallest temperatures the sum is the number of
    maxima, at the largest the number of tokens that are not masked."""
    g = torch.Generator(device="cuda").manual_seed(V)
    l = torch.randint(-4, 5, (5, V), generator=g, device="cuda").to(dtype)
    l[:, ::7] = float("-inf")
    st = _stats(tv, l, T)
    m = l.double().amax(dim=1)
    n = (l.double() == m[:, None]).sum(dim=1) if T < 1 else torch.isfinite(l).sum(dim=1)
    assert torch.equal(st[:, 0], m)
    assert float(((st[:, 1] - n).abs() / n).max()) <= 4e-6
