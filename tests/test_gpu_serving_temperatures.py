"""Temperatures whose log2(e) / T is no float32 (below 4.24e-39) are refused by the calls
that write row normalisers: with an infinite factor no weight is a number."""

import pytest
import torch

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def tv():
    import paper_2505_12398_gb300 as tv
    from paper_2505_12398_gb300.build import build
    build()
    return tv


@pytest.mark.parametrize("T", [1e-45, 1e-40, 4.2e-39])
def test_refused(tv, T):
    V = 64
    for dtype in (torch.bfloat16, torch.float32):
        v = tv.Verifier(V, 0, 2, "bf16" if dtype == torch.bfloat16 else "fp32", path="three")
        z = torch.zeros(2, 1, dtype=torch.int32, device="cuda")
        with pytest.raises(tv.LibraryError) as e:
            v.process_logits(None, z - 1, z, torch.zeros(2, 1, V, dtype=dtype, device="cuda"), T)
        assert e.value.code == -2
        v.close()
    v = tv.Verifier(V, 0, 2, "bf16", path="three")
    f8 = dict(dtype=torch.float8_e4m3fn, device="cuda")
    args = (torch.zeros(2, 16, **f8), torch.ones(2, 1, device="cuda"), torch.zeros(V, 16, **f8),
            torch.ones(1, 1, device="cuda"))
    with pytest.raises(tv.LibraryError) as e:
        v.lm_head_fp8(*args, temperature=T)
    assert e.value.code == -2
    v.close()


def test_smallest_accepted(tv):
    V = 64
    v = tv.Verifier(V, 0, 2, "bf16", path="three")
    f8 = dict(dtype=torch.float8_e4m3fn, device="cuda")
    args = (torch.zeros(2, 16, **f8), torch.ones(2, 1, device="cuda"), torch.zeros(V, 16, **f8),
            torch.ones(1, 1, device="cuda"))
    _, st = v.lm_head_fp8(*args, temperature=4.25e-39)
    assert st.tolist() == [[0.0, float(V)]] * 2
    z = torch.zeros(2, 1, dtype=torch.int32, device="cuda")
    _, st = v.process_logits(None, z - 1, z, torch.zeros(2, 1, V, dtype=torch.bfloat16,
                                                         device="cuda"), 4.25e-39)
    assert st.view(2, 2).tolist() == [[0.0, float(V)]] * 2
    v.close()
