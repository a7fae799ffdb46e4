"""The LM head on e4m3 operands with block scales (tv_lm_head_scaled) against float64.

Tolerances.  Operands k with |k| <= 8 and scales of 1/2, 1 and 2 make every product and
partial sum exact in float32, so the stored bf16 logits equal the oracle's bit for bit.
With general operands and scales a logit is within half a bf16 step plus 2^-16 of the
sum of the magnitudes of its products (float32 accumulation loses at most about 2^-24 of
that per step, K / 16 steps and a scale's rounding at most; a dropped, repeated or
misplaced block of K, or a neighbouring block's scale, is off by far more).  Normalisers
are held to the oracle's of the stored logits: the maximum equal, the sum within 1e-5."""

import numpy as np
import pytest
import torch

from oracle import lmhead, serving

pytestmark = pytest.mark.gpu

SHAPES = [
    # rows, K, V: one and few rows, a partial last group of K, one column tile and less
    (1, 16, 8), (1, 128, 128), (3, 144, 40), (16, 256, 1000), (61, 272, 1003), (128, 128, 4099),
    # pairs of SMs: more than one row tile, ragged ones
    (129, 128, 257), (200, 400, 5000), (257, 2048, 1001), (300, 640, 33), (700, 512, 32000),
    # more tiles than SMs, wide and ragged; a long K
    (40, 384, 60008), (640, 256, 60007), (5, 16384, 300),
]


@pytest.fixture(scope="module")
def tv():
    import paper_2505_12398_gb300 as tv
    from paper_2505_12398_gb300.build import build
    build()
    return tv


def _run(tv, qa, sa, qw, sw, T):
    M, V = qa.shape[0], qw.shape[0]
    v = tv.Verifier(V, 7, (M + 7) // 8, "bf16", path="three")
    args = (qa.cuda(), sa.cuda(), qw.cuda(), sw.cuda())
    lg, st = v.lm_head_fp8(*args, temperature=T)
    alone, none = v.lm_head_fp8(*args)
    torch.cuda.synchronize()
    assert v.status() == 0 and none is None
    assert torch.equal(alone, lg)
    v.close()
    return lg.float().cpu().numpy().astype(np.float64), st.cpu().numpy().astype(np.float64)


def _check_stats(got, st, T):
    m, s = lmhead.row_stats(got, T)
    assert np.array_equal(st[:, 0], m)
    assert np.max(np.abs(st[:, 1] - s) / s) < 1e-5


@pytest.mark.parametrize("M,K,V", SHAPES)
def test_exact_operands(tv, M, K, V):
    g = torch.Generator().manual_seed(M * 7 + K + V)
    G = (K + 127) // 128
    qa = torch.randint(-8, 9, (M, K), generator=g).float()
    qw = torch.randint(-8, 9, (V, K), generator=g).float()
    sa = torch.exp2(torch.randint(-1, 2, (M, G), generator=g).float())
    sw = torch.exp2(torch.randint(-1, 2, ((V + 127) // 128, G), generator=g).float()) / 64
    got, st = _run(tv, qa.to(torch.float8_e4m3fn), sa, qw.to(torch.float8_e4m3fn), sw, 0.8)
    ref = lmhead.to_bf16(serving.scaled_logits(qa.numpy(), sa.numpy(), qw.numpy(), sw.numpy()))
    assert np.array_equal(got, ref)
    _check_stats(got, st, 0.8)


@pytest.mark.parametrize("M,K,V", [(5, 4096, 1003), (61, 272, 1003), (257, 2048, 1001),
                                   (40, 1024, 20008)])
def test_random_operands(tv, M, K, V):
    g = torch.Generator().manual_seed(M + K + V)
    G = (K + 127) // 128
    qa = (torch.randn(M, K, generator=g) * 60).clamp(-448, 448).to(torch.float8_e4m3fn)
    qw = (torch.randn(V, K, generator=g) * 60).clamp(-448, 448).to(torch.float8_e4m3fn)
    sa = torch.rand(M, G, generator=g) * 1e-2 + 1e-4
    sw = torch.rand((V + 127) // 128, G, generator=g) * 1e-3 + 1e-5
    got, st = _run(tv, qa, sa, qw, sw, 1.0)
    a, w = qa.float().numpy(), qw.float().numpy()
    exact = serving.scaled_logits(a, sa.numpy(), w, sw.numpy())
    mag = serving.scaled_logits(np.abs(a), sa.numpy(), np.abs(w), sw.numpy())
    half = np.ldexp(1.0, np.frexp(got)[1] - 9)
    assert np.all(np.abs(got - exact) <= half + 2.0 ** -16 * mag)
    _check_stats(got, st, 1.0)


def test_norm_feeds_the_head(tv):
    """rms_norm's output and quantize_weight's are the head's operands as they are."""
    M, K, V = 61, 512, 3000
    g = torch.Generator().manual_seed(9)
    x = torch.randn(M, K, generator=g).to(torch.bfloat16).cuda()
    r = torch.randn(M, K, generator=g).to(torch.bfloat16).cuda()
    nw = torch.ones(K, dtype=torch.bfloat16, device="cuda")
    W = (torch.randn(V, K, generator=g) / K ** 0.5).to(torch.bfloat16).cuda()
    v = tv.Verifier(V, 60, 1, "bf16", path="three")
    qa, sa, _ = v.rms_norm(x, nw, r)
    qw, sw = v.quantize_weight(W)
    lg, _ = v.lm_head_fp8(qa, sa, qw, sw)
    a, w = qa.float().cpu().numpy(), qw.float().cpu().numpy()
    exact = serving.scaled_logits(a, sa.cpu().numpy(), w, sw.cpu().numpy())
    mag = serving.scaled_logits(np.abs(a), sa.cpu().numpy(), np.abs(w), sw.cpu().numpy())
    got = lg.float().cpu().numpy().astype(np.float64)
    half = np.ldexp(1.0, np.frexp(got)[1] - 9)
    assert np.all(np.abs(got - exact) <= half + 2.0 ** -16 * mag)
    # and near the unquantised product: two roundings of 2^-4 at most, averaging out
    y, _ = serving.rms_norm(x.float().cpu().numpy(), r.float().cpu().numpy(),
                            nw.float().cpu().numpy(), 1e-5)
    full = y @ W.double().cpu().numpy().T
    assert np.linalg.norm(got - full) < 0.06 * np.linalg.norm(full)
    assert v.status() == 0
    v.close()


def test_no_row_reads_another(tv):
    """NaN in one row, and in one weight's row, stays there."""
    M, K, V = 200, 256, 700
    qa = torch.ones(M, K, device="cuda").to(torch.float8_e4m3fn)
    qw = torch.ones(V, K, device="cuda").to(torch.float8_e4m3fn)
    sa = torch.ones(M, 2, device="cuda")
    sw = torch.ones(6, 2, device="cuda")
    qa.view(torch.uint8)[130, 7] = 0x7F
    qw.view(torch.uint8)[699, 255] = 0x7F
    for rows in (M, 100):
        v = tv.Verifier(V, 0, rows, "bf16", path="three")
        lg, st = v.lm_head_fp8(qa[:rows].contiguous(), sa[:rows].contiguous(), qw, sw, 1.0)
        nan = torch.isnan(lg)
        want = torch.zeros(rows, V, dtype=torch.bool, device="cuda")
        want[:, 699] = True
        if rows > 130:
            want[130] = True
        assert torch.equal(nan, want)
        fine = torch.ones(rows, dtype=torch.bool, device="cuda")
        if rows > 130:
            fine[130] = False
        assert (st[fine, 0] == 256.0).all() and (st[fine, 1] == V - 1).all()
        v.close()


def test_refusals(tv):
    v = tv.Verifier(256, 0, 8, "bf16", path="three")
    f8 = dict(dtype=torch.float8_e4m3fn, device="cuda")
    qa, qw = torch.zeros(8, 64, **f8), torch.zeros(256, 64, **f8)
    sa, sw = torch.ones(8, 1, device="cuda"), torch.ones(2, 1, device="cuda")
    v.lm_head_fp8(qa, sa, qw, sw)
    for bad in ((qa.view(torch.uint8), sa, qw, sw), (qa, sa[:4], qw, sw), (qa, sa, qw[:128], sw),
                (qa, sa, qw, sw[:1]), (qa, sa.cpu(), qw, sw)):
        with pytest.raises(ValueError):
            v.lm_head_fp8(*bad)
    with pytest.raises(tv.LibraryError) as e:
        v.lm_head_fp8(qa, sa, qw, sw, temperature=0.0)
    assert e.value.code == -2
    with pytest.raises(tv.LibraryError) as e:
        v.lm_head_fp8(torch.zeros(9, 64, **f8), torch.ones(9, 1, device="cuda"), qw, sw)
    assert e.value.code == -4
    with pytest.raises(tv.LibraryError):                     # K % 16 != 0
        v.lm_head_fp8(torch.zeros(8, 40, **f8), sa, torch.zeros(256, 40, **f8), sw)
    v.close()
    v = tv.Verifier(256, 0, 8, "fp32", path="three")
    with pytest.raises(tv.LibraryError):
        v.lm_head_fp8(qa, sa, qw, sw)
    v.close()
