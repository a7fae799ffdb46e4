"""A small 4-bit cache with requests in it, for the tests of the cache and of the attention
over it."""

import numpy as np
import torch

from oracle import cache as oc


class Setup:
    """A verifier and a cache with shuffled pages for requests of given lengths."""

    def __init__(self, tv, lens, room, Hk=2, d=64, P=16, layers=1, seed=0, nodes=63, spare=3,
                 fill=0xff):
        self.v = tv.Verifier(1000, nodes, len(lens), "bf16", path="three")
        self.lens, self.room, self.Hk, self.d, self.P, self.layers = lens, room, Hk, d, P, layers
        need = [(n + room + P - 1) // P for n in lens]
        total = sum(need) + spare
        rng = np.random.default_rng(seed)
        order = rng.permutation(total)
        table = np.full((len(lens), max(need) + 1), -1, dtype=np.int32)
        at = 0
        for b, n in enumerate(need):
            table[b, :n] = order[at:at + n]
            at += n
        self.np_table = table
        self.np_exp = rng.integers(-5, 4, (layers, 2, Hk)).astype(np.int32)
        # (bytes that no row was written to are NaN scales)
        data = torch.full((layers, total, Hk, 2, P * d * 9 // 16), fill, dtype=torch.uint8,
                          device="cuda")
        self.cache = tv.KVCache(self.v, layers, total, Hk, d, page_size=P, data=data,
                                exponents=torch.from_numpy(self.np_exp).cuda())
        self.table = torch.from_numpy(table).cuda()
        self.lengths = torch.tensor(lens, dtype=torch.int32, device="cuda")
        self.g = torch.Generator().manual_seed(seed + 1)

    def rows(self, R, dtype=torch.bfloat16, spread=6.0):
        """Keys or values over many powers of two."""
        shape = (len(self.lens), R, self.Hk, self.d)
        x = torch.randn(shape, generator=self.g)
        e = torch.rand(shape[:3] + (1,), generator=self.g) * 2 * spread - spread
        return (x * torch.exp2(e)).to(dtype)

    def want(self, x, layer, side):
        """What the cache holds for rows [..., Hk, d]."""
        x = x.double().numpy()
        return np.stack([oc.held(x[..., h, :], int(self.np_exp[layer, side, h]))
                         for h in range(self.Hk)], axis=-2)

    def fill(self, layer=0, dtype=torch.bfloat16, spread=1.0, extra=0):
        """Writes every request's cached tokens (and `extra` behind them); what the cache
        then holds, [tokens, Hk, d] of each request, keys and values."""
        R = max(self.lens) + extra
        k, v = self.rows(R, dtype, spread), self.rows(R, dtype, spread)
        counts = torch.tensor([n + extra for n in self.lens], dtype=torch.int32, device="cuda")
        if R > 0:
            self.cache.write(layer, k.cuda(), v.cuda(), torch.zeros_like(self.lengths),
                             self.table, rows=counts)
        wk, wv = self.want(k, layer, 0), self.want(v, layer, 1)
        return [(wk[b, :n + extra], wv[b, :n + extra]) for b, n in enumerate(self.lens)]
