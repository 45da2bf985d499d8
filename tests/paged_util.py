"""Caches in pages for the tests, and plain 64-bit implementations of what works on them, on host tensors."""
import math

import torch

import paper_2502_04507_amd as sta
from tests import layer_util as lu

BF = torch.bfloat16
DEV = "cuda:0"


def starts(lengths):
    out = [0]
    for n in lengths:
        out.append(out[-1] + n)
    return out


def ints(x):
    return torch.tensor(x, dtype=torch.int32, device=DEV)


class Cache:
    """Sequences of `used` keys whose pages lie in the pool in any order, among pages that are nobody's.  k, v: host [used, Hkv, D] of every sequence.  What is not used
    holds NaN and infinities; entries of the table behind the last used page are no pages."""

    def __init__(self, Hkv, D, page, used, seed, layout="tokens", room=None, keys=None, spread=1.0):
        g = torch.Generator().manual_seed(seed)
        self.Hkv, self.D, self.page, self.used = Hkv, D, page, list(used)
        need = [-(-n // page) for n in used]
        self.width = max(need + [0]) + 2 if room is None else room
        self.pages = sum(need) + 3
        order = torch.randperm(self.pages, generator=g).tolist()
        self.rows, at = [], 0
        for n in need:
            self.rows.append(order[at:at + n])
            at += n
        self.k, self.v = keys or ([(torch.randn((n, Hkv, D), generator=g) * spread).to(BF) for n in used], [torch.randn((n, Hkv, D), generator=g).to(BF) for n in used])
        shape = (self.pages, page, Hkv, D)
        pool = [torch.full(shape, float("nan"), dtype=BF), torch.full(shape, float("inf"), dtype=BF)]
        for s, n in enumerate(used):
            for j in range(need[s]):
                here = slice(j * page, min(n, (j + 1) * page))
                for x, y in zip(pool, (self.k[s], self.v[s])):
                    x[self.rows[s][j], :here.stop - here.start] = y[here]
        table = torch.full((len(used), self.width), 1 << 30, dtype=torch.int32)
        for s, row in enumerate(self.rows):
            table[s, :len(row)] = torch.tensor(row, dtype=torch.int32)
        if layout == "heads":                               # [pages, heads, slots, D]
            pool = [x.transpose(1, 2).contiguous().to(DEV).transpose(1, 2) for x in pool]
        elif layout == "halves":                            # keys and values of a page side by side, rows of a wider tensor
            both = torch.full((self.pages, 2, page, Hkv + 1, D + 8), 7.0, dtype=BF, device=DEV)
            pool = [both[:, i, :, :Hkv, 8:].copy_(x) for i, x in enumerate(pool)]
        else:
            pool = [x.to(DEV) for x in pool]
        self.pool = pool
        wide = torch.full((len(used), self.width + 3), -1, dtype=torch.int32, device=DEV)
        wide[:, :self.width] = table.to(DEV)
        self.table, self.lengths = wide[:, :self.width], ints(self.used)
        self.sta = sta.StaPagedCache(pool[0], pool[1], self.table, self.lengths)

    def place(self, s, j):
        return self.rows[s][j // self.page], j % self.page


def forward(q, cache, new, causal=True, scale=0.0, lse=False, workspace=True, max_k=None, o=None):
    """q: device [tokens, Hq, D]; returns o and lse."""
    o = torch.full_like(q, 7.0) if o is None else o
    lse = torch.full((q.shape[1], q.shape[0]), 7.0, device=DEV) if lse else None
    max_q, max_k = max(new), max(cache.used) if max_k is None else max_k
    n = sta.sta_paged_workspace_bytes(q.shape[1], cache.Hkv, cache.D, len(new), q.shape[0], max_q, max_k) if workspace else 0
    ws = torch.full((max(n, 16),), 255, dtype=torch.uint8, device=DEV) if workspace else None
    sta.sta_paged_forward(q, o, ints(starts(new)), cache.sta, max_q, max_k, causal=causal, scale=scale, lse=lse, workspace=ws)
    return o, lse


def packed(q, cache, new, causal=True, scale=0.0, lse=False, workspace=True):
    """The same of the keys side by side, through sta_packed_forward."""
    k, v = (torch.cat(x).to(DEV) for x in (cache.k, cache.v))
    o = torch.full_like(q, 7.0)
    lse = torch.full((q.shape[1], q.shape[0]), 7.0, device=DEV) if lse else None
    max_q, max_k = max(new), max(cache.used)
    n = sta.sta_packed_workspace_bytes(q.shape[1], cache.Hkv, cache.D, len(new), q.shape[0], max_q, max_k) if workspace else 0
    ws = torch.full((max(n, 16),), 255, dtype=torch.uint8, device=DEV) if workspace else None
    sta.sta_packed_forward(q, k, v, o, ints(starts(new)), ints(starts(cache.used)), max_q, max_k, causal=causal, scale=scale, lse=lse, workspace=ws)
    return o, lse


def same(a, b):
    return torch.equal(a.contiguous().view(torch.int16 if a.dtype == BF else torch.int32), b.contiguous().view(torch.int16 if b.dtype == BF else torch.int32))


def weights(q, k, lse, causal, scale):
    """One sequence: what every key gathers, [Hkv, lk], from the rows' given lse [Hq, lq]; all float64.  Rows without keys give nothing."""
    lq, Hq, _ = q.shape
    lk, Hkv = k.shape[0], k.shape[1]
    keep = lu.seen(lq, lk, causal)
    w = torch.zeros((Hkv, lk), dtype=torch.float64)
    for h in range(Hq):
        n = h // (Hq // Hkv)
        p = torch.where(keep, torch.exp(q[:, h] @ k[:, n].T * scale - lse[h][:, None]), 0.0)
        w[n] += torch.where((lse[h] == -math.inf)[:, None], 0.0, p).sum(0)
    return w


def survivors(w, keep, first, recent):
    """Indices that stay of n weights, ascending."""
    n = len(w)
    if n <= keep:
        return list(range(n))
    middle = sorted(range(first, n - recent), key=lambda j: (-w[j], j))[:keep - first - recent]
    return sorted(list(range(first)) + middle + list(range(n - recent, n)))
