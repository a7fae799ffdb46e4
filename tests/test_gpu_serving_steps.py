"""The steps beside verification at the sizes where their launch shapes and offsets change:
every tile width of the 8-bit LM head (on one SM and on pairs), arrays whose offsets pass
2^31 elements, CUDA graphs, calls from several threads, and the whole cycle of
workloads/serve_cycle.py."""

import threading

import numpy as np
import pytest
import torch

from oracle import lmhead, serving

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def tv():
    import paper_2505_12398_gb300 as tv
    from paper_2505_12398_gb300.build import build
    build()
    return tv


def _operands(M, K, V, seed):
    """e4m3 whole numbers up to 8 with scales 1/2, 1 and 2: every sum is exact."""
    g = torch.Generator(device="cuda").manual_seed(seed)
    G = (K + 127) // 128
    qa = torch.randint(-8, 9, (M, K), generator=g, device="cuda").float()
    qw = torch.randint(-8, 9, (V, K), generator=g, device="cuda").float()
    sa = torch.exp2(torch.randint(-1, 2, (M, G), generator=g, device="cuda").float())
    sw = torch.exp2(torch.randint(-1, 2, ((V + 127) // 128, G), generator=g, device="cuda")
                    .float()) / 64
    return qa, sa, qw, sw


def _rows_of(qa, sa, qw, sw, rows):
    """The exact logits of some rows, in float64 on the GPU."""
    k = torch.arange(qa.shape[1], device="cuda") // 128
    v = torch.arange(qw.shape[0], device="cuda") // 128
    a = qa[rows].double() * sa[rows].double()[:, k]
    return a @ (qw.double() * sw.double()[v][:, k]).T


@pytest.mark.parametrize("M,V", [(40, 20000), (40, 25000), (40, 30000), (40, 35000), (128, 17408),
                                 (300, 5000), (300, 7000), (300, 8000), (300, 9600),
                                 (520, 14003), (130, 19464)])
def test_every_tile_width(tv, M, V):
    K = 320
    qa, sa, qw, sw = _operands(M, K, V, M + V)
    v = tv.Verifier(V, 0, M, "bf16", path="three")
    lg, st = v.lm_head_fp8(qa.to(torch.float8_e4m3fn), sa, qw.to(torch.float8_e4m3fn), sw, 0.9)
    want = _rows_of(qa, sa, qw, sw, slice(None)).float().to(torch.bfloat16)
    assert torch.equal(lg, want)
    m, s = lmhead.row_stats(want.double().cpu().numpy(), 0.9)
    st = st.double().cpu().numpy()
    assert np.array_equal(st[:, 0], m) and np.max(np.abs(st[:, 1] - s) / s) < 1e-5
    assert v.status() == 0
    v.close()


@pytest.mark.parametrize("M", [1, 31, 64, 129, 290])
@pytest.mark.parametrize("V", [1, 7, 33, 63, 97, 130, 991, 1012, 2045, 2046])
def test_rows_of_any_length(tv, M, V):
    """Vocabularies that are not whole 16-byte pieces, from one token on: every logit, and
    nothing written before or past them."""
    K = 144
    qa, sa, qw, sw = _operands(M, K, V, 3 * M + V)
    v = tv.Verifier(V, 0, M, "bf16", path="three")
    big = torch.full((M * V + 64,), 7.0, dtype=torch.bfloat16, device="cuda")
    out = big[32:32 + M * V].view(M, V)
    v.lm_head_fp8(qa.to(torch.float8_e4m3fn), sa, qw.to(torch.float8_e4m3fn), sw, out=(out, None))
    want = _rows_of(qa, sa, qw, sw, slice(None)).float().to(torch.bfloat16)
    assert torch.equal(out, want)
    assert bool((big[:32] == 7).all()) and bool((big[32 + M * V:] == 7).all())
    assert v.status() == 0
    v.close()


def test_head_past_32_bit_offsets(tv):
    """18000 x 128256 logits: 2.3e9 of them; rows at both ends and across the middle."""
    M, K, V = 18000, 64, 128256
    qa, sa, qw, sw = _operands(M, K, V, 3)
    v = tv.Verifier(V, 0, M, "bf16", path="three")
    lg, st = v.lm_head_fp8(qa.to(torch.float8_e4m3fn), sa, qw.to(torch.float8_e4m3fn), sw, 1.0)
    rows = torch.tensor([0, 1, 255, 256, 8999, 16743, 16744, 17919, 17920, 17999], device="cuda")
    want = _rows_of(qa, sa, qw, sw, rows).float().to(torch.bfloat16)
    assert torch.equal(lg[rows], want)
    assert torch.equal(st[rows, 0], want.float().amax(dim=1))
    assert v.status() == 0
    v.close()


@pytest.mark.parametrize("V", [128256, 128251])
def test_processing_past_32_bit_offsets(tv, V):
    """280 trees of 61 rows (2.2e9 logits), with the contexts of slots whose arrays pass
    2^31 elements as well."""
    B, R, S = 280, 61, 17000
    v = tv.Verifier(V, R - 1, B, "bf16", path="three")
    ctx = tv.TokenContext(v, S)
    dev = v.device
    g = torch.Generator(device="cuda").manual_seed(1)
    slots = torch.arange(S - B, S, dtype=torch.int32, device=dev)
    words = torch.randint(0, V, (B, 50), generator=g, device=dev, dtype=torch.int32)
    ctx.add_generated(words, slots=slots)
    ctx.set_bias(words[:, :1].contiguous(), torch.full((B, 1), 2.0, device=dev), slots=slots)
    lg = torch.randn(B, R, V, generator=g, device=dev, dtype=torch.float32).to(torch.bfloat16) \
        if V == 128256 else torch.empty(B, R, V, dtype=torch.bfloat16, device=dev).normal_(
            generator=g)
    par = torch.arange(-1, R - 1, dtype=torch.int32, device=dev).expand(B, R).contiguous()
    tok = torch.randint(0, V, (B, R), generator=g, device=dev, dtype=torch.int32)
    pen = torch.tensor([[1.25, 0.5, 0.25]], device=dev).expand(B, 3).contiguous()
    res, st = v.process_logits(ctx, par, tok, lg, 1.0, slots=slots, penalties=pen)
    assert v.status() == 0
    for b, i in ((0, 0), (0, 60), (140, 3), (274, 30), (279, 0), (279, 60)):
        counts = (ctx.counts[S - B + b] >> 1).cpu().numpy()
        want = serving.process_row(lg[b, i].float().cpu().numpy(), counts, None,
                                   ctx.bias[S - B + b].cpu().numpy(), (1.25, 0.5, 0.25),
                                   serving.path_tokens(par[b].tolist(), tok[b].tolist(), i), None)
        got = res[b, i].double().cpu().numpy()
        half = np.ldexp(1.0, np.frexp(got)[1] - 9)
        assert np.all(np.abs(got - want) <= half + 2.0 ** -20 * (1 + np.abs(want)))
        m, s = serving.row_normaliser(got, 1.0)
        assert float(st[b, i, 0]) == m and abs(float(st[b, i, 1]) - s) <= 2e-6 * s
    v.close()


def test_graph_replays(tv):
    """Norm, head, processing and the context's update captured once and replayed on new
    inputs give what the eager calls give."""
    M, K, V, B = 32, 256, 1024, 4
    R = M // B
    v = tv.Verifier(V, R - 1, B, "bf16")
    dev = v.device
    g = torch.Generator(device="cuda").manual_seed(2)
    qw, sw = v.quantize_weight(torch.randn(V, K, generator=g, device=dev).to(torch.bfloat16))
    nw = torch.ones(K, dtype=torch.bfloat16, device=dev)
    x = torch.randn(M, K, generator=g, device=dev).to(torch.bfloat16)
    r = torch.randn(M, K, generator=g, device=dev).to(torch.bfloat16)
    par = torch.tensor([-1] + [0] * (R - 1), dtype=torch.int32, device=dev).expand(B, R).contiguous()
    tok = torch.randint(0, V, (B, R), generator=g, device=dev, dtype=torch.int32)
    pen = torch.full((B, 3), 1.5, device=dev)

    def step(ctx):
        q, s, _ = v.rms_norm(x, nw, r)
        lg, _ = v.lm_head_fp8(q, s, qw, sw, temperature=0.8)
        res, st = v.process_logits(ctx, par, tok, lg.view(B, R, V), 0.8, penalties=pen)
        ctx.add_generated(tok)
        return res, st

    ctx, eager = tv.TokenContext(v, B), tv.TokenContext(v, B)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step(tv.TokenContext(v, B))
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        res, st = step(ctx)
    ctx.counts.zero_()
    ctx.marks.zero_()
    for k in range(3):
        x.copy_(torch.randn(M, K, generator=g, device=dev))
        tok.copy_(torch.randint(0, V, (B, R), generator=g, device=dev))
        graph.replay()
        a, b = step(eager)
        assert torch.equal(res, a) and torch.equal(st, b)
        assert torch.equal(ctx.counts, eager.counts) and torch.equal(ctx.marks, eager.marks)
    assert v.status() == 0
    v.close()


def test_handles_in_several_threads(tv):
    """Four threads, each with its own handle and stream, get what one alone gets."""
    M, K, V = 200, 384, 3000
    qa, sa, qw, sw = _operands(M, K, V, 11)
    qa8, qw8 = qa.to(torch.float8_e4m3fn), qw.to(torch.float8_e4m3fn)
    want = _rows_of(qa, sa, qw, sw, slice(None)).float().to(torch.bfloat16)
    z = torch.zeros(M, 1, dtype=torch.int32, device="cuda")
    bad = []
    torch.cuda.synchronize()

    def work():
        try:
            st = torch.cuda.Stream()
            v = tv.Verifier(V, 0, M, "bf16", path="three")
            for _ in range(5):
                lg, rs = v.lm_head_fp8(qa8, sa, qw8, sw, 1.0, stream=st)
                res, ps = v.process_logits(None, z - 1, z, lg.view(M, 1, V), 1.0, stream=st)
                st.synchronize()
                ok = torch.equal(lg, want) and torch.equal(res.view(M, V), want) and \
                    torch.equal(ps.view(M, 2)[:, 0], rs[:, 0]) and \
                    torch.allclose(ps.view(M, 2)[:, 1], rs[:, 1], rtol=2e-6, atol=0.0)
                if not ok:
                    bad.append("differs")
            v.close()
        except Exception as e:      # noqa: BLE001
            bad.append(repr(e))

    threads = [threading.Thread(target=work) for _ in range(4)]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    assert not bad, bad


def test_the_cycle(tv):
    """The example's texts obey its grammar and its counts are its texts'."""
    from workloads import serve_cycle
    out = serve_cycle.run(batch=6, vocab=2048, hidden=256, cycles=5, seed=4)
    assert out["status"] & ~16 == 0
    for b, text in enumerate(out["texts"]):
        assert len(text) >= 5
        for prev, cur in zip([out["prompts"][b][-1]] + text[:-1], text):
            assert serve_cycle.allowed(prev, cur)
        counts = np.bincount(text, minlength=2048)
        assert np.array_equal(out["counts"][b] >> 1, counts)
        seen = np.bincount(out["prompts"][b], minlength=2048) > 0
        assert np.array_equal((out["counts"][b] & 1) == 1, seen)
    assert out["accepted"] > 0
