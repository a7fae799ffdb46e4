"""The 8-bit LM head on single SMs where rows are not whole 16-byte pieces and a tile has
more than 128 columns: exact operands, so every logit equals the exact one."""

import numpy as np
import pytest
import torch

from oracle import lmhead

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def tv():
    import paper_2505_12398_gb300 as tv
    from paper_2505_12398_gb300.build import build
    build()
    return tv


# tiles of 160, 192, 224 and 256 columns on 152 SMs
@pytest.mark.parametrize("M,V", [(40, 20003), (128, 25001), (1, 25006), (40, 30005), (128, 34999),
                                 (77, 34993), (1, 30011)])
def test_wide_tiles_of_one_sm(tv, M, V):
    K = 272
    g = torch.Generator(device="cuda").manual_seed(M + V)
    G = (K + 127) // 128
    qa = torch.randint(-8, 9, (M, K), generator=g, device="cuda").float()
    qw = torch.randint(-8, 9, (V, K), generator=g, device="cuda").float()
    sa = torch.exp2(torch.randint(-1, 2, (M, G), generator=g, device="cuda").float())
    sw = torch.exp2(torch.randint(-1, 2, ((V + 127) // 128, G), generator=g, device="cuda")
                    .float()) / 64
    k = torch.arange(K, device="cuda") // 128
    want = ((qa.double() * sa.double()[:, k]) @
            (qw.double() * sw.double()[torch.arange(V, device="cuda") // 128][:, k]).T)
    want = want.float().to(torch.bfloat16)
    v = tv.Verifier(V, 0, M, "bf16", path="three")
    args = (qa.to(torch.float8_e4m3fn), sa, qw.to(torch.float8_e4m3fn), sw)
    big = torch.full((M * V + 64,), 7.0, dtype=torch.bfloat16, device="cuda")
    out = big[32:32 + M * V].view(M, V)
    v.lm_head_fp8(*args, out=(out, None))
    assert torch.equal(out, want)
    assert bool((big[:32] == 7).all()) and bool((big[32 + M * V:] == 7).all())
    lg, st = v.lm_head_fp8(*args, temperature=0.9)
    assert torch.equal(lg, want)
    m, s = lmhead.row_stats(want.double().cpu().numpy(), 0.9)
    st = st.double().cpu().numpy()
    assert np.array_equal(st[:, 0], m) and np.max(np.abs(st[:, 1] - s) / s) < 1e-5
    assert v.status() == 0
    v.close()
