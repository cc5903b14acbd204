"""A key/value cache in pages, filled on the CPU, with what attention over it gives in 64 bits; shares
no code with the package."""
import math

import torch

from tests.window_reference import HALF_STEP, attention

BF16, FP32 = torch.bfloat16, torch.float32


class Cache:
    """Pages of random tokens for sequences of `own` tokens behind a common prefix.  What no token lies in
    is NaN and infinity.  order: "heads" [pages, h, T, D], "tokens" [pages, T, h, D] or "gaps" (a part
    of wider pages).  bad: (sequence or -1 for the prefix, index) of table entries that name no page."""

    def __init__(self, gen, dtype, kv, T, D, own, prefix=0, order="heads", bad=(), width=None, spare=2):
        self.kv, self.T, self.D, self.own, self.prefix = kv, T, D, list(own), prefix
        need = [-(-n // T) for n in own]
        shared = -(-prefix // T)
        self.width = max(need + [1]) if width is None else width
        self.pages = shared + sum(need) + spare
        ids = torch.randperm(self.pages, generator=gen).tolist()
        self.prefix_table, at = ids[:shared], shared
        self.table = []
        for n in need:
            # entries behind the last page: no page, or any
            rest = [(-1, 1 << 30, 0)[i % 3] for i in range(self.width - n)]
            self.table.append(ids[at:at + n] + rest)
            at += n
        k = torch.full((self.pages, kv, T, D), float("nan"), dtype=dtype)
        v = torch.full((self.pages, kv, T, D), float("inf"), dtype=dtype)
        for tokens, row in [(prefix, self.prefix_table)] + list(zip(own, self.table)):
            for i in range(-(-tokens // T)):
                n = min(T, tokens - i * T)
                for x in (k, v):
                    x[row[i], :, :n] = torch.randn(kv, n, D, generator=gen).to(dtype)
        self.k64, self.v64 = k.double(), v.double()
        self.hidden = set(bad)
        names_none = [-1, self.pages, -(1 << 31), (1 << 31) - 1]
        self.true_prefix_table, self.true_table = list(self.prefix_table), [list(r) for r in self.table]
        for x, (b, i) in enumerate(bad):
            (self.prefix_table if b < 0 else self.table[b])[i] = names_none[x % 4]
        self.k, self.v = (self._lay(x, order) for x in (k, v))

    def _lay(self, x, order):
        if order == "heads":
            return x.cuda()
        if order == "tokens":
            return x.transpose(1, 2).contiguous().cuda().transpose(1, 2)
        wide = torch.full((self.pages, self.kv + 1, self.T + 3, self.D + 8), float("nan"), dtype=x.dtype)
        wide[:, 1:, 2:-1, :-8] = x
        return wide.cuda()[:, 1:, 2:-1, :-8]

    def tables(self):
        return (torch.tensor(self.table, dtype=torch.int32).cuda(),
                torch.tensor(self.prefix_table, dtype=torch.int32).cuda() if self.prefix else None)

    def sequence(self, b, kl, prefix):
        """(k, v) [kv, tokens, D] in 64 bits and which tokens have a page."""
        page, row, there = [], [], []
        for who, tokens, names in ((-1, prefix, self.true_prefix_table), (b, kl, self.true_table[b])):
            for i in range(-(-tokens // self.T)):
                n = min(self.T, tokens - i * self.T)
                page += [names[i]] * n
                row += range(n)
                there += [(who, i) not in self.hidden] * n
        k, v = (x[page, :, row].transpose(0, 1) for x in (self.k64, self.v64))
        there = torch.tensor(there, dtype=torch.bool)
        return k, v, there


def check(cache, q64, out, lse, q_lens, k_lens, prefix, dtype, left=-1, sinks=0, scale=0.0):
    """out, lse of [B, h, N, D] queries in 64 bits on the CPU; returns the worst share of the bounds."""
    B, h, N, D = q64.shape
    G = h // cache.kv
    sc = scale if scale > 0.0 else 1.0 / math.sqrt(D)
    worst = 0.0
    for b in range(B):
        ql, kl = min(max(q_lens[b], 0), N), min(max(k_lens[b], 0), cache.width * cache.T)
        k, v, there = cache.sequence(b, kl, prefix)
        i, j = torch.arange(N).unsqueeze(1), torch.arange(prefix + kl).unsqueeze(0)
        p = prefix + kl - ql + i
        see = (i < ql) & (j <= p) & there
        if left >= 0:
            see = see & ((j >= p - left) | (j < sinks))
        for a in range(h):
            if prefix + kl == 0:
                r = {"out": torch.zeros(N, D), "lse": torch.full((N,), -math.inf)}
                assert torch.equal(out[b, a], r["out"].double()) and torch.equal(lse[b, a], r["lse"].double())
                continue
            qq = torch.where(i < ql, q64[b, a], torch.zeros_like(q64[b, a]))
            r = attention(qq, k[a // G], v[a // G], see, sc)
            for x, ref, tol in ((out[b, a], r["out"], r["out_tol"](dtype)), (lse[b, a], r["lse"], r["lse_tol"])):
                d = (x - ref).abs()
                share = torch.where(x == ref, torch.zeros_like(d), d / tol)
                worst = max(worst, float(share.max()))
                assert bool((share <= 1.0).all()), f"sequence {b}, head {a}: {float(share.max())} of the bound"
    return worst


def strided(x, memory):
    """The CPU tensor x [B, h, N, D] on the GPU with some memory order."""
    if memory == "heads":
        return x.cuda()
    if memory == "tokens":
        return x.transpose(1, 2).contiguous().cuda().transpose(1, 2)
    B, h, N, D = x.shape
    wide = torch.full((B, N + 1, h + 2, D + 8), float("nan"), dtype=x.dtype)
    wide[:, 1:, 1:1 + h, :D] = x.transpose(1, 2)
    return wide.cuda()[:, 1:, 1:1 + h, :D].transpose(1, 2)
