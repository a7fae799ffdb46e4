"""Performance cases of a 4-bit key/value cache and of the attention of drafted trees over it:

    attend   attention of every row of a batch of trees (or of causal rows) over a paged
             cache held in 4 bits: a row sees the request's cached tokens, its ancestors in
             the tree and itself
    store    keys and values quantised as they are written, and those rows read back
    read     a stretch of the cache read back
    cycle    one layer's part of a decoding cycle: the tree's rows written, attended, the
             accepted path's rows moved behind the root, and what the cache then holds there

Cache format: e2m1 codes with one e4m3 scale for each 16 columns of a row and a power of two
for each head.  A page holds page_size tokens; its block for one head's keys (or values) has
the codes [head_dim / 32][page_size][16 bytes] (column 2j of 32 in the low half of byte j)
and then the scales [head_dim / 32][page_size][2].  Tree shapes are those of the
repository's workloads; heads, pages and lengths are generic.
"""

import math

import torch

own = False

LEVELS = (0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0)      # magnitudes of the codes 0..7

# Tree shapes: nodes per level and most children per node of a level; "one" is the
# root alone, a decoding step without drafts.
SHAPES = {
    "one": ((), ()),
    "chain8": ((1,) * 8, (1,) * 8),
    "binary4": ((2, 4, 8, 16), (2, 2, 2, 2)),
    "tree26": ((2, 4, 8, 8, 4), (2, 2, 2, 1, 1)),
    "tree60": ((4, 10, 16, 16, 8, 6), (4, 3, 2, 2, 1, 1)),
    "tree120": ((4, 12, 24, 24, 20, 16, 12, 8), (4, 3, 2, 1, 1, 1, 1, 1)),
}


def _parents(shape):
    levels, most = SHAPES[shape]
    parents, prev = [-1], [0]
    for size, k in zip(levels, most):
        cur = []
        for j in range(size):
            parents.append(prev[j // k])
            cur.append(len(parents) - 1)
        prev = cur
    return parents


def _depth(parents, i):
    n = 0
    while parents[i] >= 0:
        i = parents[i]
        n += 1
    return n


def _case(name, call, batch, ctx, tree="one", rows=0, kv_heads=8, group=4, dim=128, page=64,
          dtype="bf16"):
    """rows > 0: causal rows (a piece of a prompt), rows of the longest request; else a tree."""
    return {"name": name, "call": call, "batch": batch, "ctx": ctx, "tree": tree, "rows": rows,
            "kv_heads": kv_heads, "group": group, "dim": dim, "page": page, "dtype": dtype}


def listed():
    return [
        # one token of one request: launch and latency count
        _case("attend_one_b1_2k", "attend", 1, 2000),
        # a serving batch without drafts: the cache's bytes count
        _case("attend_one_b128_8k", "attend", 128, 8192),
        # a small tree, heads of their own, a short head dimension, small pages
        _case("attend_tree26_b32_3k_d64", "attend", 32, 3001, "tree26", kv_heads=16, group=1,
              dim=64, page=16),
        # a long document, one request
        _case("attend_tree60_b1_128k", "attend", 1, 131000, "tree60"),
        # a serving batch of trees
        _case("attend_tree60_b128_4k", "attend", 128, 4096, "tree60"),
        # pieces of prompts behind what is cached of them
        _case("attend_prompt_b8_777", "attend", 8, 1500, rows=777, page=128),
        # one request's tree; prompts of a batch
        _case("store_tree60_b1", "store", 1, 4000, "tree60"),
        _case("store_prompt_b16_2k", "store", 16, 0, rows=2048),
        # a stretch of one request; whole requests in fp32
        _case("read_b1_1000", "read", 1, 1000, page=16),
        _case("read_b32_4k_fp32", "read", 32, 4096, dtype="fp32"),
        # one layer of one request's cycle; of a serving batch
        _case("cycle_chain8_b1_2k", "cycle", 1, 2000, "chain8"),
        _case("cycle_tree26_b64_4k", "cycle", 64, 4096, "tree26", group=8),
    ]


# No drawn case costs more than the largest listed one of its call: query rows times cached
# tokens, and rows, of a head of 128 columns.
MOST_SCORES = 128 * 61 * 4096 * 32
MOST_CACHED = 128 * 8192 * 8
MOST_ROWS = 16 * 2048 * 8


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(max(lo, hi))))))


def draw(rng):
    call = rng.choice(["attend", "attend", "attend", "store", "read", "cycle"])
    kv_heads, group = rng.choice([1, 2, 4, 8, 8, 16]), rng.choice([1, 2, 3, 4, 4, 5, 8, 16])
    dim, page = rng.choice([64, 128, 128]), rng.choice([16, 32, 64, 64, 128])
    dtype = "bf16" if call in ("attend", "cycle") else rng.choice(["bf16", "fp32"])
    tree, rows = rng.choice(sorted(SHAPES)), 0
    if call in ("attend", "store") and rng.random() < 0.3:
        rows = _log_int(rng, 2, 2048)
    if call == "cycle" and tree == "one":
        tree = "chain8"
    R = rows or len(_parents(tree))
    ctx = _log_int(rng, 1, 131072)
    if call == "read":
        most = MOST_ROWS // (ctx * kv_heads)
        if most < 1:
            ctx, most = MOST_ROWS // kv_heads, 1
    else:
        most = min(MOST_SCORES // (R * (ctx + R) * kv_heads * group),
                   MOST_CACHED // ((ctx + R) * kv_heads), MOST_ROWS // (R * kv_heads))
        while most < 1:
            ctx //= 2
            most = min(MOST_SCORES // (R * (ctx + R) * kv_heads * group),
                       MOST_CACHED // ((ctx + R) * kv_heads), MOST_ROWS // (R * kv_heads))
    return {"call": call, "batch": _log_int(rng, 1, min(256, most)), "ctx": ctx, "tree": tree,
            "rows": rows, "kv_heads": kv_heads, "group": group, "dim": dim, "page": page,
            "dtype": dtype}


def _sizes(case):
    """(rows of the longest request, cached tokens and rows of each request): the lengths
    lie between half of the longest and all of it."""
    B, R = case["batch"], case["rows"] or len(_parents(case["tree"]))
    lens = [case["ctx"] - (b * 7919) % (case["ctx"] // 2 + 1) for b in range(B)]
    rows = [R - (b * 104729) % (R // 2 + 1) if case["rows"] else R for b in range(B)]
    return R, lens, rows


# --------------------------------------------------------------------- inputs


def _generator(seed):
    return torch.Generator(device="cuda").manual_seed(seed)


def _torch_dtype(name):
    return torch.bfloat16 if name == "bf16" else torch.float32


def _keys(shape, dtype, g):
    """Keys or values: normal, with a few columns of every head larger than the rest."""
    x = torch.randn(shape, generator=g, device="cuda")
    loud = torch.rand(shape[-2:], generator=g, device="cuda") < 0.02
    return torch.where(loud, 8.0 * x, x).to(dtype)


def _inputs(case, seed):
    """The cache with its page table, the new rows, and the accepted paths."""
    g = _generator(seed)
    R, lens, rows = _sizes(case)
    B, Hk, d, P = case["batch"], case["kv_heads"], case["dim"], case["page"]
    dev, dtype = "cuda", _torch_dtype(case["dtype"])
    need = [(n + R + P - 1) // P for n in lens]
    table = torch.full((B, max(need)), -1, dtype=torch.int32)
    total = sum(need)
    order = torch.randperm(total, generator=g, device=dev).cpu().to(torch.int32)
    at = 0
    for b, n in enumerate(need):
        table[b, :n] = order[at:at + n]
        at += n
    exponents = torch.randint(-4, 1, (1, 2, Hk), generator=g, device=dev, dtype=torch.int32)
    # what is cached: codes of normal values (scaled by the largest of 16) and their scales
    data = torch.empty(1, total, Hk, 2, P * d * 9 // 16, dtype=torch.uint8, device=dev)
    step = max(1, (1 << 26) // (Hk * 2 * P * d))
    for p in range(0, total, step):
        x = _keys((min(step, total - p), Hk, 2, P, d), torch.float32, g)
        data[0, p:p + step] = _encode(x, exponents[0].T[None])
    s = {"case": case, "call": case["call"], "lens": lens, "rows": rows, "data": data,
         "exponents": exponents, "table": table.to(dev), "R": R,
         "lengths": torch.tensor(lens, dtype=torch.int32, device=dev),
         "row_counts": torch.tensor(rows, dtype=torch.int32, device=dev)}
    parents = [-1] + list(range(R - 1)) if case["rows"] else _parents(case["tree"])
    s["parents"] = parents
    s["parents_dev"] = torch.tensor(parents, dtype=torch.int32, device=dev).expand(B, R) \
        .contiguous()
    ancestors = torch.tril(torch.ones(R, R, dtype=torch.bool))
    if not case["rows"]:
        ancestors = torch.eye(R, dtype=torch.bool)
        for i in range(1, R):
            ancestors[i] |= ancestors[parents[i]]
    s["ancestors"] = ancestors.to(dev)
    if case["call"] in ("attend", "cycle"):
        s["q"] = torch.randn(B, R, Hk * case["group"], d, generator=g, device=dev).to(dtype)
    if case["call"] in ("store", "cycle"):
        s["k"] = _keys((B, R, Hk, d), dtype, g)
        s["v"] = _keys((B, R, Hk, d), dtype, g)
    if case["call"] == "cycle":
        # paths to random nodes; now and then a tree that was found invalid
        ends = torch.randint(0, R, (B,), generator=g, device=dev).tolist()
        path = torch.full((B, R - 1), -1, dtype=torch.int32)
        tau = []
        for b, i in enumerate(ends):
            chain = []
            while i > 0:
                chain.append(i)
                i = parents[i]
            if b % 16 == 15:
                tau.append(-1)
                continue
            path[b, :len(chain)] = torch.tensor(chain[::-1], dtype=torch.int32)
            tau.append(len(chain))
        s["paths"], s["taus"] = path.tolist(), tau
        s["path"] = path.to(dev)
        s["tau"] = torch.tensor(tau, dtype=torch.int32, device=dev)
        s["deepest"] = 1 + max(_depth(parents, i) for i in range(R))
    return s


def prepare(case, seed):
    s = _inputs(case, seed)
    if own:      # the library's handle, and the cache around the same arrays
        import paper_2505_12398_gb300 as tv
        s["verifier"] = tv.Verifier(1024, s["R"] - 1 if not case["rows"] else 0, case["batch"],
                                    "bf16", path="three")
        s["cache"] = tv.KVCache(s["verifier"], 1, s["data"].shape[1], case["kv_heads"],
                                case["dim"], page_size=case["page"], data=s["data"],
                                exponents=s["exponents"])
    return s


# ----------------------------------------------------------------------- runs


def _run_own(s):
    cache, case = s["cache"], s["case"]
    at = (s["lengths"], s["table"])
    counts = s["row_counts"] if case["rows"] else None
    parents = None if case["rows"] else s["parents_dev"]
    if s["call"] == "attend":
        return cache.attend(0, s["q"], *at, parents=parents, rows=counts)
    if s["call"] == "store":
        cache.write(0, s["k"], s["v"], *at, rows=counts)
        return cache.read(0, s["lengths"] + s["row_counts"], s["table"], s["R"],
                          first=s["lengths"], dtype=case["dtype"])
    if s["call"] == "read":
        return cache.read(0, *at, case["ctx"], dtype=case["dtype"])
    cache.write(0, s["k"], s["v"], *at)
    out = cache.attend(0, s["q"], *at, parents=parents)
    lengths = cache.accept(s["path"], s["tau"], *at)
    k, v = cache.read(0, lengths, s["table"], s["deepest"], first=s["lengths"],
                      dtype=case["dtype"])
    return out, lengths, k, v


def _round_scale(x):
    """The e4m3 values nearest to x >= 0 (64 bits), ties to even."""
    _, e = torch.frexp(x)
    step = torch.exp2((e - 1).clamp(min=-6).double() - 3.0)
    return (torch.round(x / step) * step).clamp(max=448.0)


def _encode(x, exponents):
    """The bytes [..., P * d * 9 / 16] of rows x [..., heads, 2, P, d] with exponents
    [..., heads, 2].  The borders between codes are compared in 64 bits."""
    P, d = x.shape[-2:]
    y = x.double() * torch.exp2(-exponents.double())[..., None, None]
    y = y.reshape(*y.shape[:-1], d // 16, 16)
    scale = _round_scale(y.abs().amax(dim=-1) / 6.0)
    a, t = y.abs(), scale[..., None]
    code = torch.zeros_like(a, dtype=torch.uint8)
    for k in range(7):
        border = (LEVELS[k] + LEVELS[k + 1]) / 2 * t
        code += (a > border) if k % 2 == 0 else (a >= border)      # ties to the even code
    code *= t > 0
    code = torch.where((y < 0) & (code > 0), code + 8, code)
    code = code.reshape(*code.shape[:-2], d // 32, 16, 2)
    packed = code[..., 0] | (code[..., 1] << 4)                    # [..., P, d / 32, 16]
    packed = packed.transpose(-3, -2).flatten(-3)
    s8 = scale.float().to(torch.float8_e4m3fn).view(torch.uint8)
    s8 = s8.reshape(*s8.shape[:-1], d // 32, 2).transpose(-3, -2).flatten(-3)
    return torch.cat([packed, s8], dim=-1)


def _decode(data, exponents, P, d):
    """Values [..., heads, 2, P, d] in 32 bits of the bytes [..., heads, 2, P * d * 9 / 16]."""
    codes = data[..., :P * d // 2].reshape(*data.shape[:-1], d // 32, P, 16)
    table = torch.tensor(LEVELS + tuple(-x for x in LEVELS), device=data.device)
    x = torch.stack([table[(codes & 15).long()], table[(codes >> 4).long()]], dim=-1)
    x = x.flatten(-2).transpose(-3, -2).flatten(-2)                # [..., P, d]
    s = data[..., P * d // 2:].contiguous().view(torch.float8_e4m3fn).float()
    s = s.reshape(*data.shape[:-1], d // 32, P, 2).transpose(-3, -2).flatten(-2)
    return x * s.repeat_interleave(16, dim=-1) * torch.exp2(exponents.float())[..., None, None]


def _cached(s, b, first, last):
    """Keys and values [heads, 2, last - first, d] of a request's positions."""
    case, P = s["case"], s["case"]["page"]
    lo, hi = first // P, (last + P - 1) // P
    pages = s["table"][b, lo:hi].long()
    x = _decode(s["data"][0, pages], s["exponents"][0].T[None], P, case["dim"])
    x = x.permute(1, 2, 0, 3, 4).flatten(2, 3)
    return x[:, :, first - lo * P:last - lo * P]


def _plain_attend(s):
    case, q = s["case"], s["q"]
    B, R, H, d = q.shape
    Hk = case["kv_heads"]
    out = torch.zeros(B, R, H, d, dtype=q.dtype, device=q.device)
    for b in range(B):
        n, r = s["lens"][b], s["rows"][b]
        x = _cached(s, b, 0, n + r)
        qb = q[b, :r].float().reshape(r, Hk, H // Hk, d).permute(1, 2, 0, 3).flatten(1, 2)
        t = (qb @ x[:, 0].transpose(1, 2)) * (1.0 / math.sqrt(d))
        t = t.reshape(Hk, H // Hk, r, n + r)
        t[..., n:].masked_fill_(~s["ancestors"][:r, :r], -math.inf)
        t = torch.exp(t - t.amax(dim=-1, keepdim=True))
        o = (t / t.sum(dim=-1, keepdim=True)).flatten(1, 2) @ x[:, 1]
        out[b, :r] = o.reshape(Hk, H // Hk, r, d).permute(2, 0, 1, 3).reshape(r, H, d).to(q.dtype)
    return out


def _plain_write(s):
    case, P, d = s["case"], s["case"]["page"], s["case"]["dim"]
    whole = s["data"][0]
    for b in range(case["batch"]):
        n, r = s["lens"][b], s["rows"][b]
        x = torch.stack([s["k"][b, :r], s["v"][b, :r]], dim=2)     # [r, heads, 2, d]
        new = _encode(x[..., None, :], s["exponents"][0].T[None])  # pages of one row
        pos = torch.arange(n, n + r, device="cuda")
        page, slot = s["table"][b].long()[pos // P], pos % P
        half = d // 2
        codes = whole[..., :P * half].view(*whole.shape[:-1], d // 32, P, 16)
        codes[page, :, :, :, slot] = new[..., :half].reshape(*new.shape[:-1], d // 32, 16)
        scales = whole[..., P * half:].view(*whole.shape[:-1], d // 32, P, 2)
        scales[page, :, :, :, slot] = new[..., half:].reshape(*new.shape[:-1], d // 32, 2)


def _plain_read(s, firsts, lasts, n, dtype):
    case = s["case"]
    shape = (case["batch"], n, case["kv_heads"], case["dim"])
    k = torch.zeros(shape, dtype=dtype, device="cuda")
    v = torch.zeros(shape, dtype=dtype, device="cuda")
    for b in range(case["batch"]):
        m = min(lasts[b] - firsts[b], n)
        if m > 0:
            x = _cached(s, b, firsts[b], firsts[b] + m).permute(1, 2, 0, 3).to(dtype)
            k[b, :m], v[b, :m] = x[0], x[1]
    return k, v


def _plain_accept(s):
    """Moves the accepted rows of every request; the new lengths."""
    case, P, d = s["case"], s["case"]["page"], s["case"]["dim"]
    whole = s["data"][0]
    codes = whole[..., :P * d // 2].view(*whole.shape[:-1], d // 32, P, 16)
    scales = whole[..., P * d // 2:].view(*whole.shape[:-1], d // 32, P, 2)
    for b, tau in enumerate(s["taus"]):
        if tau > 0:
            n = s["lens"][b]
            src = n + s["path"][b, :tau].long()
            dst = n + 1 + torch.arange(tau, device="cuda")
            table = s["table"][b].long()
            for a in (codes, scales):
                a[table[dst // P], :, :, :, dst % P] = a[table[src // P], :, :, :, src % P]
    return torch.where(s["tau"] >= 0, s["lengths"] + 1 + s["tau"], s["lengths"])


def run(state):
    if own:
        return _run_own(state)
    s, case = state, state["case"]
    dtype = _torch_dtype(case["dtype"])
    if s["call"] == "attend":
        return _plain_attend(s)
    if s["call"] == "store":
        _plain_write(s)
        return _plain_read(s, s["lens"], [n + r for n, r in zip(s["lens"], s["rows"])], s["R"],
                           dtype)
    if s["call"] == "read":
        return _plain_read(s, [0] * case["batch"], s["lens"], case["ctx"], dtype)
    _plain_write(s)
    out = _plain_attend(s)
    lengths = _plain_accept(s)
    lasts = [n + 1 + t if t >= 0 else n for n, t in zip(s["lens"], s["taus"])]
    return (out, lengths) + _plain_read(s, s["lens"], lasts, s["deepest"], dtype)


# ----------------------------------------------------------------------- work


def work(case):
    R, lens, rows = _sizes(case)
    Hk, d = case["kv_heads"], case["dim"]
    H = Hk * case["group"]
    size = 2 if case["dtype"] == "bf16" else 4
    row, packed = 2 * Hk * d * size, 2 * Hk * d * 9 // 16          # keys and values of a token
    if case["call"] == "read":
        return {"bytes": sum(lens) * (packed + row), "flops": sum(lens) * 4 * Hk * d}
    if case["call"] == "store":
        return {"bytes": sum(rows) * (2 * row + 2 * packed), "flops": sum(rows) * 12 * Hk * d}
    parents = [-1] + list(range(R - 1)) if case["rows"] else _parents(case["tree"])
    seen = [0] * (R + 1)                 # rows of the tree that the first i rows see
    for i in range(R):
        seen[i + 1] = seen[i] + (i if case["rows"] else _depth(parents, i)) + 1
    scores = sum(n * r + seen[r] for n, r in zip(lens, rows))
    out = {"bytes": sum(n + r for n, r in zip(lens, rows)) * packed + sum(rows) * H * d * 4,
           "flops": 4 * H * d * scores}
    if case["call"] == "cycle":          # its new rows are read, written and read back
        out["bytes"] += sum(rows) * (row + packed)
    return out


# ------------------------------------------------------------ 64-bit results


def _grid16(x, exponent):
    """x [..., d] in 64 bits as the cache holds it, group by group of 16 columns."""
    out = torch.empty_like(x)
    unit = 2.0 ** exponent
    for c in range(0, x.shape[-1], 16):
        y = x[..., c:c + 16] / unit
        top = y.abs().max(dim=-1, keepdim=True).values / 6.0
        ulp = torch.exp2(torch.floor(torch.log2(top.clamp(min=2.0 ** -6))) - 3.0)
        s = torch.minimum(torch.round(top / ulp) * ulp,
                          torch.tensor(448.0, dtype=torch.float64, device="cuda"))
        r = torch.where(s > 0, y / torch.where(s > 0, s, torch.ones_like(s)),
                        torch.zeros_like(y))
        a = r.abs()
        step = torch.where(a < 2.0, 0.5, torch.where(a < 4.0, 1.0, 2.0))
        q = torch.clamp(torch.round(a / step) * step, max=6.0)
        out[..., c:c + 16] = torch.sign(r) * q * s * unit
    return out


def _held(s, b, h, which, last):
    """What head h of request b holds at positions 0 .. last - 1, in 64 bits."""
    P, d = s["case"]["page"], s["case"]["dim"]
    pos = torch.arange(last, device="cuda")
    block = s["data"][0, :, h, which].index_select(0, s["table"][b, :(last + P - 1) // P].long())
    out = torch.empty(last, d, dtype=torch.float64, device="cuda")
    page, slot = pos // P, pos % P
    unit = 2.0 ** int(s["exponents"][0, which, h])
    levels = torch.tensor(LEVELS, dtype=torch.float64, device="cuda")
    for c in range(d // 32):
        raw = block[page, :][torch.arange(last, device="cuda")[:, None],
                             ((c * P + slot) * 16)[:, None] + torch.arange(16, device="cuda")]
        for half in range(2):
            nib = (raw >> (4 * half)) & 15
            val = levels[(nib & 7).long()] * (1.0 - 2.0 * (nib >> 3).double())
            out[:, 32 * c + half:32 * c + 32:2] = val
        for k in range(2):
            byte = block[page, P * d // 2 + (c * P + slot) * 2 + k].long()
            e, m = (byte >> 3) & 15, (byte & 7).double()
            sc = torch.where(e > 0, (1.0 + m / 8.0) * torch.exp2(e.double() - 7.0),
                             m * 2.0 ** -9)
            out[:, 32 * c + 16 * k:32 * c + 16 * k + 16] *= (sc * unit)[:, None]
    return out


def exact(case, seed):
    s = _inputs(case, seed)
    B, Hk, d, R = case["batch"], case["kv_heads"], case["dim"], s["R"]
    G, call = case["group"], case["call"]
    new = {}
    if call in ("store", "cycle"):
        for name, which in (("k", 0), ("v", 1)):
            x = s[name].double()
            new[which] = torch.stack([_grid16(x[:, :, h], int(s["exponents"][0, which, h]))
                                      for h in range(Hk)], dim=2)
    if call == "store":
        on = (torch.arange(R, device="cuda")[None] < s["row_counts"][:, None])[..., None, None]
        return tuple(torch.where(on, new[w], torch.zeros_like(new[w])) for w in (0, 1))
    if call == "read":
        k, v = (torch.zeros(B, case["ctx"], Hk, d, dtype=torch.float64, device="cuda")
                for _ in range(2))
        for b in range(B):
            for h in range(Hk):
                k[b, :s["lens"][b], h] = _held(s, b, h, 0, s["lens"][b])
                v[b, :s["lens"][b], h] = _held(s, b, h, 1, s["lens"][b])
        return k, v
    out = torch.zeros(B, R, Hk * G, d, dtype=torch.float64, device="cuda")
    for b in range(B):
        n, r = s["lens"][b], s["rows"][b]
        hidden = torch.ones(r, n + r, dtype=torch.bool, device="cuda")
        hidden[:, :n] = False
        if case["rows"]:
            hidden[:, n:] = torch.triu(hidden[:, n:], diagonal=1)
        else:
            mine = [[] for _ in range(r)]
            for i in range(r):
                j = i
                while j >= 0:
                    mine[i].append(j)
                    j = s["parents"][j]
            for i in range(r):
                hidden[i, n + torch.tensor(mine[i], device="cuda")] = False
        for h in range(Hk):
            last = n if call == "cycle" else n + r
            K, V = _held(s, b, h, 0, last), _held(s, b, h, 1, last)
            if call == "cycle":
                K = torch.cat([K, new[0][b, :r, h]])
                V = torch.cat([V, new[1][b, :r, h]])
            for g in range(h * G, h * G + G):
                t = s["q"][b, :r, g].double() @ K.T / d ** 0.5
                t[hidden] = -math.inf
                out[b, :r, g] = torch.softmax(t, dim=1) @ V
    if call == "attend":
        return out
    k, v = (torch.zeros(B, s["deepest"], Hk, d, dtype=torch.float64, device="cuda")
            for _ in range(2))
    lengths = s["lengths"].clone()
    for b in range(B):
        if s["taus"][b] >= 0:
            picked = [0] + s["paths"][b][:s["taus"][b]]
            lengths[b] += len(picked)
            k[b, :len(picked)] = new[0][b, picked]
            v[b, :len(picked)] = new[1][b, picked]
    return out, lengths, k, v
