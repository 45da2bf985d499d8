"""New rows and kept rows that are more than the caches hold, which go past them, on the GPU: every bit against rows gathered by indexing, and the attention that reads them next."""
import pytest
import torch

import paper_2502_04507_amd as sta
from tests.paged_util import BF, DEV, ints, same, starts

pytestmark = pytest.mark.gpu
CACHES = 32 << 20               # bytes; a call that writes more than as much of K goes past the caches


def pages_of(lengths, page, seed, room=0):
    """A table of pages in any order, and how many pages the pool has (two of them nobody's)."""
    need = [max(-(-n // page), room) for n in lengths]
    order = torch.randperm(sum(need) + 2, generator=torch.Generator().manual_seed(seed)).to(torch.int32)
    table = torch.full((len(lengths), max(need)), -1, dtype=torch.int32)
    for s, n in enumerate(need):
        table[s, :n] = order[sum(need[:s]):sum(need[:s]) + n]
    return table.to(DEV), sum(need) + 2


def slots_of(table, s, keys, page):
    return table[s, keys // page].long() * page + keys % page


@pytest.mark.parametrize("dtype", [BF, torch.float32])
@pytest.mark.parametrize("Hq,Hkv,D,page", [(16, 8, 128, 24), (16, 16, 64, 5)])
def test_append_and_the_attention_behind_it(Hq, Hkv, D, page, dtype):
    new, before = [5000, 1, 3300, 77], [100, 3000, 0, 50]
    used, T = [a + b for a, b in zip(new, before)], sum(new)
    assert 4 * T * Hkv * D > CACHES
    g = torch.Generator(device=DEV).manual_seed(3)
    table, pages = pages_of(used, page, 4)
    pool = [torch.randn((pages, page, Hkv, D), generator=g, device=DEV).to(BF) for _ in range(2)]
    weights = torch.full((pages, Hkv, page), 3.0, device=DEV)
    x = torch.randn((T, 2 * Hkv, D), generator=g, device=DEV).to(dtype)
    cu = starts(new)
    want, want_w = [t.clone() for t in pool], weights.clone()
    for s in range(len(new)):
        at = slots_of(table, s, torch.arange(before[s], used[s], device=DEV), page)
        for i, t in enumerate(want):
            t.view(-1, Hkv, D)[at] = x[cu[s]:cu[s + 1], i * Hkv:(i + 1) * Hkv].to(BF)
        want_w[at // page, :, at % page] = 0.0
    cache = sta.StaPagedCache(*pool, table, ints(used))
    sta.sta_paged_append(x[:, :Hkv], x[:, Hkv:], ints(cu), cache, max(new), weights=weights)
    q = torch.randn((8, Hq, D), generator=g, device=DEV).to(BF)                 # the last two tokens of every sequence, straight behind
    o, o2 = torch.empty_like(q), torch.empty_like(q)
    sta.sta_paged_forward(q, o, ints([0, 2, 4, 6, 8]), cache, 2, max(used))
    assert all(same(a, b) for a, b in zip(pool, want)) and torch.equal(weights, want_w)
    rows = torch.cat([slots_of(table, s, torch.arange(n, device=DEV), page) for s, n in enumerate(used)])
    k, v = (t.view(-1, Hkv, D)[rows] for t in want)
    sta.sta_packed_forward(q, k, v, o2, ints([0, 2, 4, 6, 8]), ints(starts(used)), 2, max(used))
    assert same(o, o2)


@pytest.mark.parametrize("shared", [False, True])
@pytest.mark.parametrize("Hkv,D,page,to_page", [(8, 128, 24, 20), (16, 64, 64, 7)])
def test_evict(Hkv, D, page, to_page, shared):
    used, keep, first, recent = [9000, 2100, 4000, 2500, 100], 2100, 4, 100
    S = len(used)
    assert 4 * S * Hkv * keep * D > CACHES
    g = torch.Generator(device=DEV).manual_seed(5)
    table, pages = pages_of(used, page, 6)
    cache = sta.StaPagedCache(*[torch.randn((pages, page, Hkv, D), generator=g, device=DEV).to(BF) for _ in range(2)], table, ints(used), shared=shared)
    to_table, to_pages = pages_of([keep] * S, to_page, 7)
    into = sta.StaPagedCache(*[torch.full((to_pages, to_page, Hkv, D), 7.0, dtype=BF, device=DEV) for _ in range(2)], to_table, ints([0] * S), shared=shared)
    # numbers that all differ, so that the order needs no rule
    w = torch.randperm(cache.weights_shape[0] * Hkv * cache.weights_shape[2], generator=g, device=DEV).float().view(cache.weights_shape)
    to_w, kept = torch.full(into.weights_shape, 7.0, device=DEV), torch.zeros((S, Hkv, keep), dtype=torch.int32, device=DEV)
    sta.sta_paged_evict(cache, w, into, to_w, kept, first=first, recent=recent)
    want = [torch.full_like(t, 7.0) for t in (into.k, into.v, to_w)]
    for s, n in enumerate(used):
        at, stay = slots_of(table, s, torch.arange(n, device=DEV), page), min(n, keep)
        to = slots_of(to_table, s, torch.arange(stay, device=DEV), to_page)
        for h in range(Hkv):
            numbers = w[s, h, :n].clone() if shared else w[at // page, h, at % page]
            order = numbers.clone()
            order[:first] = order[n - recent:] = float("inf")
            j = torch.sort(torch.topk(order, stay).indices).values
            assert torch.equal(kept[s, h, :stay], j.int()) and bool((kept[s, h, stay:] == -1).all()), (s, h)
            for t, x in zip(want, (cache.k, cache.v)):
                t.view(-1, Hkv, D)[to, h] = x.view(-1, Hkv, D)[at[j], h]
            if shared:
                want[2][s, h, :stay] = numbers[j]
            else:
                want[2][to // to_page, h, to % to_page] = numbers[j]
    assert into.used.tolist() == [min(n, keep) for n in used]
    assert same(into.k, want[0]) and same(into.v, want[1]) and torch.equal(to_w, want[2])
