"""The final norm with the residual's addition (tv_rms_norm) and the quantisation of
weights (tv_quantize_weight) against float64.

Tolerances.  y in fp32: the sum of squares, its root, the division and two products
are within 2^-20 of the exact value, relative (a tree sum of at most 65536 squares
loses at most about 20 roundings of 2^-24, halved by the root).  A bf16 output is then
within half a step plus that.  An e4m3 output is the rounding of some value within
2^-18 of the exact quotient.  The residual stream is the float32 sum rounded once, and
weights have no arithmetic but the division: both are compared bit for bit."""

import numpy as np
import pytest
import torch

from oracle import serving

pytestmark = pytest.mark.gpu

DTYPES = {"bf16": torch.bfloat16, "fp32": torch.float32}


@pytest.fixture(scope="module")
def v():
    import paper_2505_12398_gb300 as tv
    from paper_2505_12398_gb300.build import build
    build()
    handle = tv.Verifier(1024, 0, 1, "bf16", path="three")
    yield handle
    handle.close()


def _np(t):
    return t.float().cpu().numpy().astype(np.float64)


def _inputs(M, K, dtype, wdtype, residual, seed):
    g = torch.Generator().manual_seed(seed)
    x = torch.randn(M, K, generator=g)
    x[:, ::97] *= 30.0
    r = torch.randn(M, K, generator=g) * 3 if residual else None
    w = 1.0 + 0.2 * torch.randn(K, generator=g)
    return (x.to(DTYPES[dtype]).cuda(), r.to(DTYPES[dtype]).cuda() if residual else None,
            w.to(DTYPES[wdtype]).cuda())


def _check(got, x, r, w, eps, quantize):
    y, _ = serving.rms_norm(_np(x), None if r is None else _np(r), _np(w), eps)
    if quantize:
        q, s, total = got
        s = s.cpu().numpy().astype(np.float64)
        want = serving.row_scales(y)
        assert s.shape == want.shape
        assert np.all(np.abs(s - want) <= 2.0 ** -20 * want)
        v = y / serving.spread(want, *y.shape, 1)
        d = 2.0 ** -18 * np.abs(v)
        q = _np(q)
        assert np.all(q >= serving.round_e4m3(v - d)) and np.all(q <= serving.round_e4m3(v + d))
    else:
        o, total = got
        o = _np(o)
        half = np.ldexp(1.0, np.frexp(o)[1] - 9)
        assert np.all(np.abs(o - y) <= half + 2.0 ** -20 * np.abs(y))
    if r is None:
        assert total is None
    else:
        h = x.float() + r.float()
        assert torch.equal(total, h.to(x.dtype))


@pytest.mark.parametrize("quantize", [True, False])
@pytest.mark.parametrize("M,K,dtype,wdtype,residual", [
    (1, 8, "bf16", "bf16", True), (3, 128, "fp32", "bf16", True), (5, 136, "bf16", "fp32", False),
    (61, 4096, "bf16", "bf16", True), (7, 4104, "bf16", "bf16", False),
    (33, 2320, "fp32", "fp32", True), (2, 8200, "bf16", "bf16", True),
    (2, 16384, "fp32", "fp32", True), (1, 40000, "bf16", "bf16", True),
    (1, 65536, "fp32", "bf16", False), (700, 1000, "bf16", "bf16", True)])
def test_norm(v, M, K, dtype, wdtype, residual, quantize):
    x, r, w = _inputs(M, K, dtype, wdtype, residual, M * 131 + K)
    _check(v.rms_norm(x, w, r, eps=1e-5, quantize=quantize), x, r, w, 1e-5, quantize)
    torch.cuda.synchronize()
    assert v.status() == 0


def test_rows_of_zeros_and_of_tiny_values(v):
    """A zero row: scales 2^-100 / 448 and zeros.  Rows far below 1 are lifted to
    magnitude sqrt(mean) / sqrt(mean + eps)."""
    x = torch.zeros(3, 256, dtype=torch.float32, device="cuda")
    x[1] = 1e-6
    x[2, 200] = 1e-3
    w = torch.ones(256, dtype=torch.float32, device="cuda")
    q, s, _ = v.rms_norm(x, w, eps=1e-5)
    assert (q[0].float() == 0).all() and (s[0] == np.float32(2.0 ** -100) / np.float32(448)).all()
    assert (q[2, :128].float() == 0).all()
    _check((q, s, None), x, None, w, 1e-5, True)


def test_nan_and_infinity_stay_in_their_group(v):
    x = torch.ones(2, 384, dtype=torch.bfloat16, device="cuda")
    w = torch.ones(384, dtype=torch.bfloat16, device="cuda")
    w[130] = float("nan")
    q, s, _ = v.rms_norm(x, w)
    assert torch.isnan(s[:, 1]).all() and torch.isnan(q[:, 130].float()).all()
    assert torch.isfinite(s[:, [0, 2]]).all() and (q[:, :128].float() == 448).all()


def test_in_place_and_streams(v):
    x, r, w = _inputs(37, 512, "bf16", "bf16", True, 5)
    want = v.rms_norm(x, w, r)
    q = torch.empty_like(want[0])
    s = torch.empty_like(want[1])
    st = torch.cuda.Stream()
    st.wait_stream(torch.cuda.current_stream())
    r2 = r.clone()
    st.wait_stream(torch.cuda.current_stream())
    v.rms_norm(x, w, r2, out=(q, s, r2), stream=st)
    st.synchronize()
    assert torch.equal(q.view(torch.uint8), want[0].view(torch.uint8))
    assert torch.equal(s, want[1]) and torch.equal(r2, want[2])
    x2 = x.clone()
    v.rms_norm(x2, w, r, out=(q, s, x2))
    assert torch.equal(x2, want[2])


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("V,K", [(1, 16), (128, 128), (129, 144), (1000, 256), (4096, 2064),
                                 (300, 16)])
def test_quantize_weight(v, V, K, dtype):
    """Scales are fl(max / 448) and values the rounding of fl(w fl(1 / s)), all IEEE
    float32 operations, so both are equal bit for bit."""
    g = torch.Generator().manual_seed(V + K)
    w = (torch.randn(V, K, generator=g) * 0.05)
    w[V // 2] = 0
    w = w.to(DTYPES[dtype])
    q, s = v.quantize_weight(w.cuda())
    wf = w.float().numpy()
    want = np.array([[np.float32(max(np.abs(wf[r:r + 128, k:k + 128]).max(),
                                     np.float32(2.0 ** -100))) / np.float32(448)
                      for k in range(0, K, 128)] for r in range(0, V, 128)], np.float32)
    assert np.array_equal(s.cpu().numpy(), want)
    inv = (np.float32(1) / want)[np.arange(V) // 128][:, np.arange(K) // 128]
    assert np.array_equal(_np(q), serving.round_e4m3(wf * inv))
    assert np.allclose(want, serving.block_scales(wf), rtol=1e-6)


def test_refusals(v):
    import paper_2505_12398_gb300 as tv
    x = torch.zeros(2, 64, dtype=torch.bfloat16, device="cuda")
    w = torch.zeros(64, dtype=torch.bfloat16, device="cuda")
    for bad in (dict(x=x[:, :60].contiguous(), weight=w[:60].contiguous()), dict(eps=0.0),
                dict(eps=float("nan"))):
        with pytest.raises(tv.LibraryError):
            v.rms_norm(**{**dict(x=x, weight=w), **bad})
    for bad in (dict(weight=w[:32]), dict(residual=x.float()), dict(x=x.half()),
                dict(x=x.t().contiguous().t()), dict(x=x.cpu()),
                dict(out=(x, None, None)), dict(residual=x, out=(None, None, None))):
        with pytest.raises((ValueError, AttributeError)):
            v.rms_norm(**{**dict(x=x, weight=w), **bad})
    with pytest.raises(tv.LibraryError):                       # not on 16 bytes
        v.rms_norm(torch.zeros(129, dtype=torch.bfloat16, device="cuda")[1:].view(2, 64), w)
    with pytest.raises(tv.LibraryError):                       # K % 16 != 0
        v.quantize_weight(torch.zeros(4, 24, dtype=torch.bfloat16, device="cuda"))
    empty = v.rms_norm(torch.zeros(0, 64, dtype=torch.bfloat16, device="cuda"), w)
    assert empty[0].shape == (0, 64)


@pytest.mark.parametrize("quantize", [True, False])
@pytest.mark.parametrize("M,K,dtype,wdtype,residual", [
    (305, 8, "bf16", "bf16", True), (1000, 128, "fp32", "bf16", True),
    (999, 256, "bf16", "fp32", False), (1001, 200, "fp32", "fp32", True),
    (4097, 248, "bf16", "bf16", True), (70001, 16, "bf16", "bf16", False),
])
def test_many_narrow_rows(v, M, K, dtype, wdtype, residual, quantize):
    x, r, w = _inputs(M, K, dtype, wdtype, residual, M + K)
    got = v.rms_norm(x, w, r, eps=1e-5, quantize=quantize)
    _check(got, x, r, w, 1e-5, quantize)
