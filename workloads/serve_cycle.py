"""A small serving program: decoding cycles of a toy target model whose last layer is in
8 bits and whose requests carry penalties, a bias and a grammar.

    python -m workloads.serve_cycle [--batch 8] [--vocab 32000] [--hidden 1024] [--cycles 20]

Each cycle drafts a tree, normalises the hidden states of its nodes (rms_norm, e4m3
output), computes their logits (lm_head_fp8), applies what the requests ask for
(process_logits: penalties for the tokens of the text and of the drafted path, biases, the
grammar's masks), verifies the tree with the normalisers that come with them
(verify_stats) and adds what was accepted to the requests' contexts (accept).  The toy
target's hidden state depends on a node's token and its parent's; the drafter is the
same model with noise.  The grammar wants token classes (t % 3) in turn 0, 1, 2, 0, ...
"""

import argparse

import torch

LEVELS = ((0, 2), (1, 2), (2, 1), (3, 1), (4, 1))   # (parent row, children) of each inner node
CLASSES = 3


def allowed(prev, cur):
    """Whether the grammar lets token ``cur`` follow ``prev``."""
    return cur % CLASSES == (prev + 1) % CLASSES


def tree_parents():
    parents = [-1]
    for parent, children in LEVELS:
        parents += [parent] * children
    return parents


def grammar_masks(vocab, device):
    """[CLASSES, ceil(vocab / 32)] int32: mask c allows the tokens of class c."""
    words = (vocab + 31) // 32
    token = torch.arange(words * 32, device=device)
    bit = torch.ones((), dtype=torch.int64, device=device) << (token % 32)
    rows = []
    for c in range(CLASSES):
        on = torch.where((token < vocab) & (token % CLASSES == c), bit, torch.zeros_like(bit))
        rows.append(on.view(words, 32).sum(dim=1))
    m = torch.stack(rows)
    return torch.where(m >= 2 ** 31, m - 2 ** 32, m).to(torch.int32)


class ToyTarget:
    """Hidden states from embeddings of a token and of the one before it, and an output
    embedding in e4m3 with block scales."""

    def __init__(self, verifier, hidden, g):
        V, dev = verifier.vocab, verifier.device
        self.emb = torch.randn(V, hidden, generator=g, device=dev).to(torch.bfloat16)
        self.before = torch.randn(V, hidden, generator=g, device=dev).to(torch.bfloat16)
        self.norm = (1 + 0.1 * torch.randn(hidden, generator=g, device=dev)).to(torch.bfloat16)
        self.head = (torch.randn(V, hidden, generator=g, device=dev) * 2.5 / hidden ** 0.5).to(
            torch.bfloat16)
        self.head8, self.scales = verifier.quantize_weight(self.head)

    def states(self, tokens, previous):
        return self.emb[tokens.long()], self.before[previous.long()]


def run(batch=8, vocab=32000, hidden=1024, cycles=20, seed=0, temperature=0.8):
    """Runs the cycles; the prompts, texts, counts, accepted drafts and the status word."""
    import paper_2505_12398_gb300 as tv

    parents = tree_parents()
    R = len(parents)
    v = tv.Verifier(vocab, R - 1, batch, "bf16")
    dev = v.device
    g = torch.Generator(device=dev).manual_seed(seed)
    target = ToyTarget(v, hidden, g)
    masks = grammar_masks(vocab, dev)
    par = torch.tensor(parents, dtype=torch.int32, device=dev).expand(batch, R).contiguous()
    up = torch.tensor([0] + parents[1:], device=dev)

    context = tv.TokenContext(v, batch)
    prompts = torch.randint(0, vocab, (batch, 12), generator=g, device=dev, dtype=torch.int32)
    context.add_prompt(prompts)
    context.set_bias(torch.full((batch, 1), vocab // 2, dtype=torch.int32, device=dev),
                     torch.full((batch, 1), 1.5, device=dev))
    penalties = torch.tensor([[1.1, 0.2, 0.1]], device=dev).expand(batch, 3).contiguous()

    last, before = prompts[:, -1].clone(), prompts[:, -2].clone()
    texts, accepted, status = [[] for _ in range(batch)], 0, 0
    for _ in range(cycles):
        # the drafted tree, level by level: rows of the nodes so far, then their children
        tokens = torch.zeros(batch, R, dtype=torch.int32, device=dev)
        tokens[:, 0] = last
        drafts = torch.zeros(batch, R, vocab, device=dev)
        u = torch.rand(batch, R, generator=g, device=dev)
        for parent, _children in LEVELS:
            prev = before if parent == 0 else tokens[:, parents[parent]]
            x, r = target.states(tokens[:, parent], prev)
            y, _ = v.rms_norm(x, target.norm, r, quantize=False)
            l = (y @ target.head.T).float() / temperature
            l += 0.3 * torch.randn(l.shape, generator=g, device=dev)
            drafts[:, parent] = torch.softmax(l, dim=-1)
            drawn = v.draft_children(par, drafts, u)
            have = par == parent
            tokens = torch.where(have, drawn, tokens)
        v.status()                # (clears it: rows that were not drafted yet had no mass)
        # the target's last layer on every node, and what the requests ask of it
        previous = torch.where(up[None] == torch.arange(R, device=dev)[None],
                               before[:, None].expand(batch, R), tokens[:, up])
        previous[:, 0] = before
        x, r = target.states(tokens.flatten(), previous.flatten())
        q, s, _ = v.rms_norm(x, target.norm, r)
        logits, _ = v.lm_head_fp8(q, s, target.head8, target.scales)
        index = ((tokens + 1) % CLASSES).to(torch.int32).contiguous()
        logits = logits.view(batch, R, vocab)
        logits, stats = v.process_logits(
            context, par, tokens, logits, temperature, penalties=penalties, masks=masks,
            mask_index=index, out=(logits, torch.empty(batch, R, 2, device=dev)))
        path, tau, bonus = v.verify_stats(
            par, tokens, logits, drafts, temperature,
            torch.rand(batch, R + 1, generator=g, device=dev), stats)
        context.accept(tokens, path, bonus)
        status |= v.status()
        # the texts, on the host
        tok, pth, bon = tokens.tolist(), path.tolist(), bonus.tolist()
        for b in range(batch):
            if bon[b] < 0:        # an invalid tree
                continue
            new = [tok[b][n] for n in pth[b] if n > 0] + [bon[b]]
            accepted += len(new) - 1
            history = prompts[b].tolist() + texts[b] + new
            texts[b] += new
            last[b], before[b] = history[-1], history[-2]
    out = {"prompts": prompts.tolist(), "texts": texts, "counts": context.counts.cpu().numpy(),
           "accepted": accepted, "status": status}
    v.close()
    return out


def main():
    ap = argparse.ArgumentParser()
    ap.add_argument("--batch", type=int, default=8)
    ap.add_argument("--vocab", type=int, default=32000)
    ap.add_argument("--hidden", type=int, default=1024)
    ap.add_argument("--cycles", type=int, default=20)
    a = ap.parse_args()
    out = run(a.batch, a.vocab, a.hidden, a.cycles)
    tokens = sum(len(t) for t in out["texts"])
    print(f"{a.cycles} cycles of {a.batch} requests: {tokens} tokens, "
          f"{out['accepted']} of them drafted ({tokens / (a.cycles * a.batch):.2f} a cycle)")


if __name__ == "__main__":
    main()
