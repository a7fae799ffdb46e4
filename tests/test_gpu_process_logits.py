"""Penalties, biases and grammar masks on tree rows (tv_process_logits) and the token
context that feeds them (tv_context_*), against float64.

Tolerances.  The arithmetic of an element is at most one division or product, one
product and three additions in float32: within 2^-22 (|l| + |l rep| + |freq n| + |pres|
+ |bias|) of the exact value, and then rounded once to the logits' type (half a step of
bf16).  Untouched elements are equal bit for bit.  Of the normaliser, which is held to
the stored values, the maximum is equal and the sum within 2e-6 (an exponential is
within 2e-7, and the sums of a thread, a warp and a row add a few 2^-24)."""

import numpy as np
import pytest
import torch

from oracle import serving

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def tv():
    import paper_2505_12398_gb300 as tv
    from paper_2505_12398_gb300.build import build
    build()
    return tv


def _bits(allowed):
    n, V = allowed.shape
    pad = np.zeros((n, (V + 31) // 32 * 32), bool)
    pad[:, :V] = allowed
    words = np.packbits(pad, axis=1, bitorder="little").view("<u4").astype(np.uint32)
    return torch.from_numpy(words.view(np.int32).copy())


def _tree(R, g, deep=False):
    return [-1] + [i - 1 if deep else int(g.integers(max(0, i - 5), i)) for i in range(1, R)]


def _case(B, R, V, dtype, seed, slots=None, n_masks=3, deep=False):
    g = np.random.default_rng(seed)
    S = B if slots is None else max(slots) + 1
    parents = [_tree(R, g, deep) for _ in range(B)]
    pool = g.integers(0, V, max(1, min(V, 40)))
    tokens = pool[g.integers(0, len(pool), (B, R))]
    # (the boundaries of words, vectors and slices)
    for k, t in enumerate((0, V - 1, 31, 32, 7, 8, 8191, 8192, 4095, 4096)):
        if t < V and R > 1:
            tokens[k % B, 1 + k % (R - 1)] = t
    generated = np.zeros((S, V), np.int64)
    prompt = np.zeros((S, V), bool)
    bias = np.zeros((S, V), np.float32)
    for s in range(S):
        np.add.at(generated[s], g.choice(np.concatenate([pool, g.integers(0, V, 60)]), 90), 1)
        prompt[s, g.integers(0, V, 50)] = True
        bias[s, g.integers(0, V, 20)] = g.normal(size=20) * 5
    allowed = g.random((n_masks, V)) < np.linspace(0.05, 0.95, n_masks)[:, None]
    if n_masks > 1:
        allowed[0] = False                    # leaves nothing
        allowed[1] = False
        allowed[1, V - 1] = True              # leaves one token
    logits = (g.normal(size=(B, R, V)) * 4).astype(np.float32)
    t = torch.from_numpy(logits).to(dtype)
    pen = np.stack([g.uniform(0.8, 1.5, B), g.uniform(-0.5, 1, B), g.uniform(-0.5, 1, B)], 1)
    return dict(B=B, R=R, V=V, S=S, parents=parents, tokens=tokens, generated=generated,
                prompt=prompt, bias=bias, allowed=allowed, logits=t,
                index=g.integers(-1, n_masks, (B, R)), pen=pen.astype(np.float32), slots=slots)


def _context(tv, v, c):
    """The context by the library's own updates: each request's texts as lists."""
    ctx = tv.TokenContext(v, c["S"])
    ctx.counts.fill_(7)                       # (cleared first)
    ctx.bias.fill_(1.0)
    ctx.marks.fill_(-1)
    dev = v.device
    ctx.clear(torch.arange(c["S"], dtype=torch.int32, device=dev))

    def ragged(rows):
        n = max(1, max(len(r) for r in rows))
        return torch.tensor([list(r) + [-1] * (n - len(r)) for r in rows], dtype=torch.int32,
                            device=dev)
    ctx.add_prompt(ragged([np.flatnonzero(p) for p in c["prompt"]]))
    ctx.add_generated(ragged([np.repeat(np.arange(c["V"]), n) for n in c["generated"]]))
    where = [np.flatnonzero(b) for b in c["bias"]]
    toks = ragged(where)
    vals = torch.zeros(toks.shape, device=dev)
    for s, w in enumerate(where):
        vals[s, :len(w)] = torch.from_numpy(c["bias"][s, w]).to(dev)
    ctx.set_bias(toks, vals)
    want = torch.from_numpy((c["generated"] * 2 + c["prompt"]).astype(np.int32)).to(dev)
    assert torch.equal(ctx.counts, want)
    assert torch.equal(ctx.bias, torch.from_numpy(c["bias"]).to(dev))
    has = (c["generated"] > 0) | c["prompt"] | (c["bias"] != 0)
    assert torch.equal(ctx.marks, _bits(has).to(dev))
    return ctx


def _run(tv, c, T=0.7, context=True, penalties=True, masks=True, in_place=False, stream=None):
    dt = "bf16" if c["logits"].dtype == torch.bfloat16 else "fp32"
    v = tv.Verifier(c["V"], c["R"] - 1, c["B"], dt, path="three")
    dev = v.device
    i32 = dict(dtype=torch.int32, device=dev)
    ctx = _context(tv, v, c) if context else None
    lg = c["logits"].to(dev)
    out = (lg.clone(), torch.empty(c["B"], c["R"], 2, device=dev)) if in_place else None
    src = out[0] if in_place else lg
    torch.cuda.synchronize()
    res, st = v.process_logits(
        ctx, torch.tensor(c["parents"], **i32), torch.tensor(c["tokens"], **i32), src, T,
        slots=None if c["slots"] is None else torch.tensor(c["slots"], **i32),
        penalties=torch.from_numpy(c["pen"]).to(dev) if penalties else None,
        masks=_bits(c["allowed"]).to(dev) if masks else None,
        mask_index=torch.tensor(c["index"], **i32) if masks else None, out=out, stream=stream)
    torch.cuda.synchronize()
    assert v.status() == 0
    v.close()
    _check(c, res, st, T, context, penalties, masks)
    return res, st


def _check(c, res, st, T, context, penalties, masks):
    got = res.float().cpu().numpy().astype(np.float64)
    stats = st.cpu().numpy().astype(np.float64)
    src = c["logits"].float().numpy().astype(np.float64)
    for b in range(c["B"]):
        s = b if c["slots"] is None else c["slots"][b]
        gen, pro, bia = (c[k][s] if context else None for k in ("generated", "prompt", "bias"))
        pen = c["pen"][b].astype(np.float64) if penalties else (1.0, 0.0, 0.0)
        for i in range(c["R"]):
            path = serving.path_tokens(c["parents"][b], c["tokens"][b], i)
            a = c["allowed"][c["index"][b, i]] if masks and c["index"][b, i] >= 0 else None
            want = serving.process_row(src[b, i], gen, pro, bia, pen, path, a)
            n = np.zeros(c["V"])
            np.add.at(n, path, 1)
            if context:
                n = n + gen
            slack = 2.0 ** -22 * (np.abs(src[b, i]) * (1 + max(pen[0], 1 / pen[0])) +
                                  abs(pen[1]) * n + abs(pen[2]) +
                                  (np.abs(bia) if context else 0))
            o = got[b, i]
            dead = np.isinf(want)
            assert np.array_equal(np.isinf(o), dead), (b, i)
            touched = (n > 0) | (pro | (bia != 0) if context else False)
            assert np.array_equal(o[~touched & ~dead], src[b, i][~touched & ~dead])
            if c["logits"].dtype == torch.bfloat16:
                slack = slack + np.ldexp(1.0, np.frexp(np.where(dead, 0, o))[1] - 9)
            assert np.all(np.abs(o - want)[~dead] <= slack[~dead]), (b, i)
            m, z = serving.row_normaliser(o, T)
            assert stats[b, i, 0] == m
            assert abs(stats[b, i, 1] - z) <= 2e-6 * z


DT = pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32], ids=["bf16", "fp32"])


@DT
@pytest.mark.parametrize("B,R,V", [
    (1, 1, 8), (2, 3, 1), (1, 4, 33), (3, 8, 1000), (2, 5, 1003), (1, 1, 32000), (2, 9, 32003),
    (1, 2, 8192), (1, 2, 8193), (1, 3, 65536), (1, 1, 128256), (1, 2, 151943), (40, 27, 520),
    (1, 1, 300001)])
def test_sizes(tv, B, R, V, dtype):
    _run(tv, _case(B, R, V, dtype, B * 31 + R + V))


@DT
@pytest.mark.parametrize("context,penalties,masks", [
    (False, False, False), (True, False, False), (False, True, False), (False, False, True),
    (True, True, False)])
def test_parts_left_out(tv, dtype, context, penalties, masks):
    _run(tv, _case(2, 6, 3001, dtype, 4), context=context, penalties=penalties, masks=masks)


@DT
@pytest.mark.parametrize("V", [4096, 4099])
def test_in_place(tv, dtype, V):
    c = _case(3, 7, V, dtype, 8)
    a, sa = _run(tv, c)
    b, sb = _run(tv, c, in_place=True)
    assert torch.equal(a, b) and torch.equal(sa, sb)


def test_slots_in_any_order(tv):
    _run(tv, _case(4, 3, 2000, torch.bfloat16, 6, slots=[5, 0, 5, 2]))


def test_deep_path(tv):
    """A chain of 1023 drafted tokens, many of them equal."""
    _run(tv, _case(1, 1024, 120, torch.float32, 2, deep=True), T=2.0)


def test_other_stream_and_temperatures(tv):
    st = torch.cuda.Stream()
    for T in (0.05, 1.0, 30.0):
        _run(tv, _case(2, 4, 5000, torch.bfloat16, 3), T=T, stream=st)


def test_masked_and_odd_logits_in(tv):
    """-inf, the type's lowest value and NaN among the logits: -inf stays, the lowest value
    weighs nothing beside the others, NaN weighs nothing and stays."""
    V = 1000
    for dtype in (torch.bfloat16, torch.float32):
        lg = torch.zeros(1, 1, V, dtype=dtype, device="cuda")
        lg[0, 0, 10:20] = float("-inf")
        lg[0, 0, 30:40] = torch.finfo(dtype).min
        lg[0, 0, 50] = float("nan")
        v = tv.Verifier(V, 0, 1, "bf16" if dtype == torch.bfloat16 else "fp32", path="three")
        z = torch.zeros(1, 1, dtype=torch.int32, device="cuda")
        res, st = v.process_logits(None, z - 1, z, lg, 1.0)
        assert torch.equal(torch.nan_to_num(res, 5.0), torch.nan_to_num(lg, 5.0))
        assert st.flatten().tolist() == [0.0, V - 21.0]
        v.close()


def test_bad_slots_masks_and_trees_are_reported(tv):
    V = 600
    v = tv.Verifier(V, 3, 2, "fp32", path="three")
    dev = v.device
    i32 = dict(dtype=torch.int32, device=dev)
    lg = torch.randn(2, 4, V, device=dev)
    par = torch.tensor([[-1, 0, 1, 0]] * 2, **i32)
    tok = torch.tensor([[0, 5, 6, 7]] * 2, **i32)
    ctx = tv.TokenContext(v, 2)
    ctx.add_generated(torch.tensor([[1], [1]], **i32))
    pen = torch.tensor([[2.0, 0.5, 0.5]] * 2, device=dev)
    masks = torch.zeros(1, (V + 31) // 32, **i32)
    idx = torch.full((2, 4), -1, **i32)

    def go(**kw):
        a = {**dict(parents=par, tokens=tok, slots=None, masks=masks, mask_index=idx), **kw}
        res, _ = v.process_logits(ctx, a["parents"], a["tokens"], lg, 1.0, slots=a["slots"],
                                  penalties=pen, masks=a["masks"], mask_index=a["mask_index"])
        return res, v.status()

    want, st = go()
    assert st == 0
    res, st = go(slots=torch.tensor([0, 2], **i32))
    assert st == 256 and torch.equal(res[0], want[0]) and res[1, 0, 1] == lg[1, 0, 1]
    bad = idx.clone()
    bad[1, 2] = 1
    res, st = go(mask_index=bad)
    assert st == 512 and torch.equal(res, want)
    bad = par.clone()
    bad[0, 2] = 3
    res, st = go(parents=bad)
    assert st & 1 and torch.equal(res[1], want[1]) and torch.equal(res[0, 1], want[0, 1])
    bad = tok.clone()
    bad[1, 1] = V
    res, st = go(tokens=bad)
    assert st & 2 and torch.equal(res[0], want[0])
    ctx.add_generated(torch.tensor([[V], [3]], **i32))
    assert v.status() == 2 and int(ctx.counts[1, 3]) == 2
    ctx.add_generated(torch.tensor([[4]], **i32), slots=torch.tensor([-1], **i32))
    assert v.status() == 256
    v.close()


def test_accept(tv):
    """The accepted path's tokens and the bonus token are counted; an invalid tree and
    padding add nothing."""
    V, N, B = 500, 5, 4
    v = tv.Verifier(V, N, B, "bf16", path="three")
    i32 = dict(dtype=torch.int32, device=v.device)
    tok = torch.tensor([[0, 11, 12, 13, 14, 15]] * B, **i32)
    path = torch.tensor([[1, 3, -1, -1, -1], [-1] * 5, [-1] * 5, [1, 2, 3, 4, 5]], **i32)
    bonus = torch.tensor([11, 499, -1, 0], **i32)
    ctx = tv.TokenContext(v, 6)
    ctx.accept(tok, path, bonus, slots=torch.tensor([5, 0, 1, 2], **i32))
    want = torch.zeros(6, V, **i32)
    want[5, 11], want[5, 13], want[0, 499] = 4, 2, 2
    want[2, [11, 12, 13, 14, 15, 0]] = 2
    assert torch.equal(ctx.counts, want) and v.status() == 0
    assert torch.equal(ctx.marks.cpu(), _bits((want > 0).cpu().numpy()))
    v.close()


def test_verification_takes_the_result(tv):
    """process_logits then verify_stats equals verify on the processed logits (decisions
    away from ties; the same normalisers up to rounding)."""
    from workloads.synth import get_workload, make_inputs
    inp = make_inputs(get_workload("eagle_v32k", batch=16), seed=5, device="cuda")
    B, R = inp.parents.shape
    V = inp.logits.shape[-1]
    v = tv.Verifier(V, R - 1, B, "bf16")
    ctx = tv.TokenContext(v, B)
    ctx.add_prompt(torch.randint(0, V, (B, 300), dtype=torch.int32, device="cuda"))
    pen = torch.tensor([[1.2, 0.2, 0.1]] * B, device="cuda")
    lg, st = v.process_logits(ctx, inp.parents, inp.tokens, inp.logits, inp.temperature,
                              penalties=pen)
    a = v.verify_stats(inp.parents, inp.tokens, lg, inp.draft_probs, inp.temperature,
                       inp.uniforms, st)
    path, tau, bonus, _, _, margin = v.verify(inp.parents, inp.tokens, lg, inp.draft_probs,
                                              inp.temperature, inp.uniforms, debug=True,
                                              margins=True)
    assert v.status() & ~16 == 0
    sure = (margin > 1e-5).all(dim=1)
    assert sure.sum() >= B // 2
    for x, y in zip(a, (path, tau, bonus)):
        assert torch.equal(x[sure], y[sure])
    v.close()


def test_a_row_left_empty_is_reported_by_verification(tv):
    V = 512
    v = tv.Verifier(V, 1, 2, "bf16")
    i32 = dict(dtype=torch.int32, device=v.device)
    par, tok = torch.tensor([[-1, 0]] * 2, **i32), torch.tensor([[0, 3]] * 2, **i32)
    lg = torch.zeros(2, 2, V, dtype=torch.bfloat16, device=v.device)
    masks = torch.zeros(1, V // 32, **i32)
    idx = torch.tensor([[0, 0], [-1, -1]], **i32)
    lg, st = v.process_logits(None, par, tok, lg, 1.0, masks=masks, mask_index=idx)
    assert st[0].tolist() == [[float("-inf"), 0.0]] * 2
    drafts = torch.full((2, 2, V), 1.0 / V, device=v.device)
    u = torch.full((2, 3), 0.5, device=v.device)
    _, tau, bonus = v.verify_stats(par, tok, lg, drafts, 1.0, u, st)
    assert v.status() & 64
    assert int(tau[0]) == -1 and int(bonus[0]) == -1 and int(tau[1]) >= 0
    v.close()


def test_refusals(tv):
    v = tv.Verifier(64, 2, 2, "bf16", path="three")
    i32 = dict(dtype=torch.int32, device=v.device)
    par = torch.tensor([[-1, 0, 0]] * 2, **i32)
    lg = torch.zeros(2, 3, 64, dtype=torch.bfloat16, device=v.device)
    ctx = tv.TokenContext(v, 1)
    with pytest.raises(tv.LibraryError):                  # two requests, one slot
        v.process_logits(ctx, par, par, lg, 1.0)
    for T in (0.0, float("inf"), -1.0):
        with pytest.raises(tv.LibraryError) as e:
            v.process_logits(None, par, par, lg, T)
        assert e.value.code == -2
    big = torch.zeros(3, 3, **i32)
    with pytest.raises(tv.LibraryError) as e:
        v.process_logits(None, big, big, torch.zeros(3, 3, 64, dtype=torch.bfloat16,
                                                     device=v.device), 1.0)
    assert e.value.code == -4
    m = torch.zeros(1, 2, **i32)
    for kw in (dict(masks=m), dict(mask_index=par), dict(masks=m[:, :1], mask_index=par),
               dict(penalties=torch.ones(2, 2, device=v.device)),
               dict(slots=torch.zeros(2, dtype=torch.int64, device=v.device)),
               dict(out=(lg.float(), None))):
        with pytest.raises(ValueError):
            v.process_logits(None, par, par, lg, 1.0, **kw)
    with pytest.raises(ValueError):
        v.process_logits(None, par, par, lg.float(), 1.0)
    other = tv.Verifier(65, 0, 1, "bf16", path="three")
    with pytest.raises(ValueError):
        other.process_logits(ctx, par[:1, :1].contiguous(), par[:1, :1].contiguous(),
                             torch.zeros(1, 1, 65, dtype=torch.bfloat16, device=v.device), 1.0)
    with pytest.raises(tv.LibraryError):                  # not on 16 bytes
        flat = torch.zeros(2 * 3 * 64 + 1, dtype=torch.bfloat16, device=v.device)
        v.process_logits(None, par, par, flat[1:].view(2, 3, 64), 1.0)
    other.close()
    v.close()
