"""Verification with the normalisers given at vocabularies that are not a multiple of 8:
what tv_process_logits and tv_lm_head_scaled write for them is taken by
tv_verify_batch_stats, which decides as tv_verify_batch does on the same logits.

Decisions are compared where the margins that the kernels themselves report exceed 1e-5:
the two calls' rates differ by their normalisers' error (2e-6 at most, 1e-7 as it goes)."""

import numpy as np
import pytest
import torch

from workloads.synth import Workload, make_inputs

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def tv():
    import paper_2505_12398_gb300 as tv
    from paper_2505_12398_gb300.build import build
    build()
    return tv


def _compare(v, inp, logits, stats):
    args = (inp.parents, inp.tokens, logits, inp.draft_probs, inp.temperature, inp.uniforms)
    path, tau, bonus, node_p, counts = v.verify_stats(*args, stats, debug=True)
    p, t, y, q, _, margin = v.verify(*args, debug=True, margins=True)
    torch.cuda.synchronize()
    assert v.status() & ~16 == 0
    assert (counts[:, 4] == 0).all()             # no row was normalised by the call
    B = tau.shape[0]
    sure = margin[:, 0] > 1e-5
    assert int(sure.sum()) >= (B + 1) // 2
    assert torch.equal(path[sure], p[sure]) and torch.equal(tau[sure], t[sure])
    both = sure & (margin[:, 1] > 1e-5)
    assert torch.equal(bonus[both], y[both]) and bool(both.any())
    assert torch.equal(torch.isnan(node_p[sure]), torch.isnan(q[sure]))
    assert torch.allclose(torch.nan_to_num(node_p[sure]), torch.nan_to_num(q[sure]), rtol=1e-3,
                          atol=1e-5)


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("V,B", [(1003, 1), (1003, 300), (32003, 32), (128251, 12), (513, 7)])
def test_processed_logits_into_verification(tv, V, B, dtype):
    w = Workload("odd", B, V, levels=(3, 5, 4), branching=(3, 2, 1), sigma=1.0)
    inp = make_inputs(w, seed=V + B, device="cuda")
    R = inp.parents.shape[1]
    logits = inp.logits.to(torch.bfloat16 if dtype == "bf16" else torch.float32)
    v = tv.Verifier(V, R - 1, B, dtype)
    ctx = tv.TokenContext(v, B)
    g = torch.Generator(device="cuda").manual_seed(3)
    ctx.add_prompt(torch.randint(0, V, (B, 200), generator=g, dtype=torch.int32, device="cuda"))
    pen = torch.tensor([[1.2, 0.2, 0.1]], device="cuda").expand(B, 3).contiguous()
    out, stats = v.process_logits(ctx, inp.parents, inp.tokens, logits, inp.temperature,
                                  penalties=pen)
    _compare(v, inp, out, stats)
    v.close()


@pytest.mark.parametrize("V,B", [(1003, 20), (32003, 8)])
def test_scaled_head_into_verification(tv, V, B):
    K = 256
    w = Workload("odd8", B, V, levels=(3, 5, 4), branching=(3, 2, 1), sigma=1.0)
    inp = make_inputs(w, seed=V, device="cuda")
    R = inp.parents.shape[1]
    g = torch.Generator(device="cuda").manual_seed(5)
    v = tv.Verifier(V, R - 1, B, "bf16")
    x = torch.randn(B * R, K, generator=g, device="cuda").to(torch.bfloat16)
    q, s, _ = v.rms_norm(x, torch.ones(K, dtype=torch.bfloat16, device="cuda"))
    W, ws = v.quantize_weight((torch.randn(V, K, generator=g, device="cuda") * 0.2)
                              .to(torch.bfloat16))
    logits, stats = v.lm_head_fp8(q, s, W, ws, temperature=inp.temperature)
    _compare(v, inp, logits.view(B, R, V), stats)
    v.close()


def test_a_row_without_a_normaliser_is_reported(tv):
    V, B = 515, 3
    v = tv.Verifier(V, 1, B, "fp32")
    i32 = dict(dtype=torch.int32, device=v.device)
    par, tok = torch.tensor([[-1, 0]] * B, **i32), torch.tensor([[0, 3]] * B, **i32)
    masks = torch.zeros(1, (V + 31) // 32, **i32)
    idx = torch.full((B, 2), -1, **i32)
    idx[1] = 0
    lg, st = v.process_logits(None, par, tok, torch.zeros(B, 2, V, device=v.device), 1.0,
                              masks=masks, mask_index=idx)
    drafts = torch.full((B, 2, V), 1.0 / V, device=v.device)
    u = torch.full((B, 3), 0.5, device=v.device)
    _, tau, bonus = v.verify_stats(par, tok, lg, drafts, 1.0, u, st)
    assert v.status() & 64
    assert int(tau[1]) == -1 and int(bonus[1]) == -1
    assert int(tau[0]) >= 0 and int(tau[2]) >= 0
    v.close()


@pytest.mark.parametrize("path", ["three", "cluster"])
def test_handles_made_for_other_paths_refuse(tv, path):
    V = 515
    v = tv.Verifier(V, 1, 1, "fp32", path=path)
    z = dict(dtype=torch.int32, device=v.device)
    par, tok = torch.tensor([[-1, 0]], **z), torch.tensor([[0, 3]], **z)
    lg = torch.zeros(1, 2, V, device=v.device)
    st = torch.tensor([[[0.0, float(V)]] * 2], device=v.device)
    with pytest.raises(tv.LibraryError) as e:
        v.verify_stats(par, tok, lg, torch.full((1, 2, V), 1.0 / V, device=v.device), 1.0,
                       torch.full((1, 3), 0.5, device=v.device), st)
    assert e.value.code == -1
    v.close()


def test_the_serving_cycle_at_an_odd_vocabulary(tv):
    from workloads import serve_cycle
    V = 2051
    out = serve_cycle.run(batch=5, vocab=V, hidden=256, cycles=4, seed=4)
    assert out["status"] & ~16 == 0
    for b, text in enumerate(out["texts"]):
        assert len(text) >= 4
        for prev, cur in zip([out["prompts"][b][-1]] + text[:-1], text):
            assert serve_cycle.allowed(prev, cur)
        assert np.array_equal(out["counts"][b] >> 1, np.bincount(text, minlength=V))
