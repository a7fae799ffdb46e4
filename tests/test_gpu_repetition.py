"""The repetition penalty as include/tv.h defines it, l / repetition for a positive logit
and l * repetition for the others, each one float32 operation: with no other penalty and no
bias the result is that of IEEE arithmetic bit for bit (rounded once more to bf16)."""

import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def tv():
    import paper_2505_12398_gb300 as tv
    from paper_2505_12398_gb300.build import build
    build()
    return tv


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32], ids=["bf16", "fp32"])
@pytest.mark.parametrize("V,share", [(40, 1.0), (3001, 1.0), (3001, 0.02), (33003, 0.05)])
def test_division_and_product(tv, V, share, dtype):
    reps = np.array([1.1, 0.7, 1.0, 1.3, 3.0, 1e30, 1e-30, 2e38, 3e-39], np.float32)
    B = len(reps)
    g = torch.Generator().manual_seed(V)
    logits = (torch.randn(B, 1, V, generator=g) * 5).to(dtype)
    on = torch.rand(B, V, generator=g) < share
    v = tv.Verifier(V, 0, B, "bf16" if dtype == torch.bfloat16 else "fp32", path="three")
    ctx = tv.TokenContext(v, B)
    n = int(on.sum(dim=1).max())
    prompt = torch.full((B, n), -1, dtype=torch.int32)
    for b in range(B):
        t = torch.nonzero(on[b]).flatten()
        prompt[b, :len(t)] = t.to(torch.int32)
    ctx.add_prompt(prompt.cuda())
    pen = torch.zeros(B, 3)
    pen[:, 0] = torch.from_numpy(reps)
    z = torch.zeros(B, 1, dtype=torch.int32, device="cuda")
    res, _ = v.process_logits(ctx, z - 1, z, logits.cuda(), 1.0, penalties=pen.cuda())
    assert v.status() == 0
    v.close()
    l = logits.float().numpy()[:, 0]
    with np.errstate(over="ignore"):
        want = np.where(l > 0, l / reps[:, None], l * reps[:, None]).astype(np.float32)
    want = torch.from_numpy(np.where(on.numpy(), want, l)).to(dtype)
    assert torch.equal(res[:, 0].cpu(), want)
