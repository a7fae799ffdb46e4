"""A context's counts and biases count only where its marks say so: include/tv.h takes a
token without its bit to have none, wherever in a row it lies and whatever the arrays hold
behind it (a slot may be emptied by its marks alone, its counts never written)."""

import pytest
import torch

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def tv():
    import paper_2505_12398_gb300 as tv
    from paper_2505_12398_gb300.build import build
    build()
    return tv


def _bits(on):
    """[n, V] truth values as [n, ceil(V / 32)] int32."""
    n, V = on.shape
    words = (V + 31) // 32
    pad = torch.zeros(n, words * 32, dtype=torch.int64, device=on.device)
    pad[:, :V] = on
    w = (pad.view(n, words, 32) << torch.arange(32, device=on.device)).sum(dim=2)
    return torch.where(w >= 2 ** 31, w - 2 ** 32, w).to(torch.int32)


def _tree(B, R, V, g):
    """A chain and a fan: the path's tokens at both ends of the row and inside it, some of
    them twice."""
    half = R // 2
    parents = [-1] + list(range(half)) + [0] * (R - 1 - half)
    ends = [x for k in range(8) for x in (k, V - 1 - k) if 0 <= x < V]
    inside = torch.randint(0, V, (B, R), generator=g)
    pick = torch.tensor(ends)[torch.randint(0, len(ends), (B, R), generator=g)]
    tokens = torch.where(torch.rand(B, R, generator=g) < 0.5, inside, pick)
    return (torch.tensor(parents, dtype=torch.int32).expand(B, R).contiguous().cuda(),
            tokens.to(torch.int32).cuda())


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32], ids=["bf16", "fp32"])
@pytest.mark.parametrize("B,R,V", [(2, 17, 40), (3, 19, 1003), (2, 33, 4096), (2, 21, 32003),
                                   (40, 27, 32003), (2, 12, 151943)])
@pytest.mark.parametrize("share", [0.0, 0.5])
def test_a_token_without_its_mark_has_no_count_and_no_bias(tv, B, R, V, dtype, share):
    """Equal to the same marks over arrays that are zero wherever a mark is missing; with no
    mark at all, also to a call without a context."""
    g = torch.Generator().manual_seed(B * 1009 + R + V)
    parents, tokens = _tree(B, R, V, g)
    counts = torch.randint(0, 40, (B, V), generator=g, dtype=torch.int32).cuda()
    bias = (torch.randn(B, V, generator=g) * 5).cuda()
    on = (torch.rand(B, V, generator=g) < share).cuda()
    v = tv.Verifier(V, R - 1, B, "bf16" if dtype == torch.bfloat16 else "fp32", path="three")
    marks = _bits(on)
    dirty = tv.TokenContext(v, B, counts=counts, bias=bias, marks=marks)
    clean = tv.TokenContext(v, B, counts=counts * on, bias=torch.where(on, bias, 0.0 * bias),
                            marks=marks)
    logits = (torch.randn(B, R, V, generator=g) * 4).to(dtype).cuda()
    pen = torch.tensor([[1.25, 0.5, 0.25]]).expand(B, 3).contiguous().cuda()
    res, st = v.process_logits(dirty, parents, tokens, logits, 0.7, penalties=pen)
    want, wst = v.process_logits(clean, parents, tokens, logits, 0.7, penalties=pen)
    assert torch.equal(res, want) and torch.equal(st, wst)
    if share == 0.0:
        want, wst = v.process_logits(None, parents, tokens, logits, 0.7, penalties=pen)
        assert torch.equal(res, want) and torch.equal(st, wst)
    assert v.status() == 0
    v.close()
