"""Sequences that share pages, with numbers of the keys by sequence, on the GPU: the same calls on copies of those pages that nobody shares, whose numbers lie beside them, give
the same bits."""
import pytest
import torch

import paper_2502_04507_amd as sta
from tests import paged_util as pu
from tests.paged_util import BF, DEV, Cache, forward, ints, same, starts
from tests.test_gpu_packed import randn
from tests.test_gpu_paged_edges import Step
from tests.test_gpu_paged_weights import gathered

pytestmark = pytest.mark.gpu


def common_beginning(Hkv, D, page, used, common, seed=9):
    """Sequences whose first `common` pages hold the same rows: every one with copies of its own, and all with the first one's."""
    g = torch.Generator().manual_seed(seed)
    keys = [[torch.randn((n, Hkv, D), generator=g).to(BF) for n in used] for _ in range(2)]
    for x in keys:
        for t in x[1:]:
            n = min(common * page, len(t), used[0])
            t[:n] = x[0][:n]
    own = Cache(Hkv, D, page, used, seed=seed, keys=keys)
    table = own.table.clone()
    for s, n in enumerate(used):
        m = min(common, n // page)              # whole pages
        table[s, :m] = own.table[0, :m]
    return own, sta.StaPagedCache(*own.pool, table, own.lengths, shared=True)


def by_sequence(own, w, fill):
    """Numbers that lie beside own's pages in the layout of a shared cache; `fill` where there is no key."""
    out = torch.full((len(own.used), own.Hkv, own.sta.room), fill, dtype=torch.float32)
    for s, n in enumerate(own.used):
        out[s, :, :n] = gathered(own, s, w).float()
    return out.to(DEV)


# Hq, Hkv, D, page, pages in common, new, used: few rows, stages by one, two and four groups, rounds of tiles
SHARED = [
    (4, 2, 128, 16, 5, [1, 2, 1], [200, 150, 96]),
    (8, 2, 64, 5, 30, [8, 8], [200, 150]),
    (4, 2, 64, 16, 5, [60, 90], [200, 150]),
    (6, 3, 128, 1, 70, [70, 45, 300], [170, 145, 301]),
    (16, 16, 64, 24, 20, [64] * 5, [1000, 999, 600, 1000, 481]),
    (16, 16, 128, 64, 130, [40, 40], [8400, 8330]),
]


@pytest.mark.parametrize("case", SHARED, ids=[str(i) for i in range(len(SHARED))])
def test_weights(case):
    """Added up in place over several calls, of rows that differ: what one sequence gives to a key of a shared page counts for it alone, and the decay once a call."""
    Hq, Hkv, D, page, common, new, used = case
    own, shared = common_beginning(Hkv, D, page, used, common)
    assert shared.weights_shape == (len(used), Hkv, shared.room) and own.sta.weights_shape == (own.pages, Hkv, page)
    w = torch.rand((own.pages, Hkv, page), generator=torch.Generator().manual_seed(2)).to(DEV)
    ws = by_sequence(own, w, 7.0)
    for seed in range(3):
        print(case, seed, flush=True)
        q = randn((sum(new), Hq, D), seed).to(DEV)
        _, lse = forward(q, own, new, lse=True)
        for cache, x in ((own.sta, w), (shared, ws)):
            sta.sta_paged_weights(q, lse, x, ints(starts(new)), cache, max(new), max(used), before=x, decay=0.75)
        assert same(ws, by_sequence(own, w, 7.0))
    # out of place, twice, by the general path as well
    out = [torch.full_like(ws, 7.0) for _ in range(2)]
    for x, stream in zip(out, (None, torch.cuda.current_stream())):
        assert sta.sta_paged_weights(q, lse, x, ints(starts(new)), shared, max(new), max(used), before=ws, decay=0.75, stream=stream) is x
    sta.sta_paged_weights(q, lse, w, ints(starts(new)), own.sta, max(new), max(used), before=w, decay=0.75)
    assert same(*out) and same(out[0], by_sequence(own, w, 7.0))


@pytest.mark.parametrize("shared_into", [False, True])
@pytest.mark.parametrize("Hkv,D,page,common,used,keep", [
    (2, 128, 16, 5, [300, 250, 90, 0], 64), (2, 64, 7, 20, [300, 250, 141], 150), (3, 128, 4, 100, [900, 850], 400), (1, 64, 64, 600, [40000, 39000], 1000), (2, 64, 1, 600, [12000, 700], 300),
])
def test_evict(Hkv, D, page, common, used, keep, shared_into):
    """Few rows in one launch and more in two, lengths beyond what a workgroup's LDS holds, pages and rows of numbers that are no multiple of four."""
    own, shared = common_beginning(Hkv, D, page, used, common)
    w = torch.randn((own.pages, Hkv, page), generator=torch.Generator().manual_seed(3)).exp().to(DEV)
    S, need = len(used), -(-keep // page)
    results = []
    for cache, x, is_shared in ((own.sta, w, False), (shared, by_sequence(own, w, 7.0), shared_into)):
        k, v = (torch.zeros((S * need, page, Hkv, D), dtype=BF, device=DEV) for _ in range(2))
        into = sta.StaPagedCache(k, v, torch.randperm(S * need, generator=torch.Generator().manual_seed(4)).view(S, need).to(torch.int32).to(DEV), ints([0] * S), shared=is_shared)
        to_w, kept = torch.full(into.weights_shape, 7.0, device=DEV), torch.zeros((S, Hkv, keep), dtype=torch.int32, device=DEV)
        for _ in range(2):
            sta.sta_paged_evict(cache, x, into, to_w, kept, first=2, recent=keep // 4)
        rows = into.table.long()
        stay = into.used.tolist()
        numbers = to_w if is_shared else to_w[rows].permute(0, 2, 1, 3).flatten(2, 3)
        results.append((k, v, kept, into.used, [numbers[s, :, :n].clone() for s, n in enumerate(stay)]))
        assert bool((numbers[0, :, stay[0]:] == 7.0).all())
    a, b = results
    assert all(torch.equal(x, y) for x, y in zip(a[:4], b[:4])) and all(torch.equal(x, y) for x, y in zip(a[4], b[4]))
    for s, n in enumerate(used):                # and by the definition
        given = gathered(own, s, w)
        for h in range(Hkv):
            assert b[2][s, h, :min(n, keep)].tolist() == pu.survivors(given[h].tolist(), keep, 2, keep // 4)


@pytest.mark.parametrize("page", [16, 5])
def test_a_run_of_all_of_them(page):
    """A prompt in common, whose pages two sequences have, continued by each; what was gathered decides what either keeps, and they go on from there."""
    Hq, Hkv, D, common, S, keep = 8, 2, 64, 4, 2, 40
    g = torch.Generator().manual_seed(21)
    width = 12 + 80 // page
    pages = 2 * S * width

    def caches(share):
        k, v = (torch.full((pages, page, Hkv, D), float("nan"), dtype=BF, device=DEV) for _ in range(2))
        table = torch.arange(pages // 2, dtype=torch.int32).view(S, width)
        behind = table + pages // 2
        table = table.clone()
        if share:
            table[1, :common] = table[0, :common]
        return [sta.StaPagedCache(k, v, t.to(DEV), ints([0] * S), shared=share) for t in (table, behind)]

    own, shared = caches(False), caches(True)
    numbers = [[torch.full(c.weights_shape, float("nan"), device=DEV) for c in cs] for cs in (own, shared)]
    # by page the two tables lie in one pool, whose numbers are one array
    numbers[0][1] = numbers[0][0]
    kept = [torch.zeros((S, Hkv, keep), dtype=torch.int32, device=DEV) for _ in range(2)]
    now = 0
    prompt = torch.randn((common * page, 2 * Hkv, D), generator=g).to(BF).to(DEV)
    for step, new in enumerate([[common * page] * 2, [7, 20], [1, 1], None, [1, 1], [3, 1]]):
        if new is None:
            for cs, ns, kp in zip((own, shared), numbers, kept):
                sta.sta_paged_evict(cs[0], ns[0], cs[1], ns[1], kp, first=1, recent=8)
            now = 1
            assert torch.equal(*kept)
            continue
        T = sum(new)
        x = torch.cat([prompt, prompt]) if step == 0 else torch.randn((T, 2 * Hkv, D), generator=g).to(BF).to(DEV)
        q = torch.randn((T, Hq, D), generator=g).to(BF).to(DEV)
        outs = []
        for cs, ns in zip((own, shared), numbers):
            cache, w, cu = cs[now], ns[now], ints(starts(new))
            cache.used.add_(ints(new))
            sta.sta_paged_append(x[:, :Hkv], x[:, Hkv:], cu, cache, max(new), weights=w)
            o, lse = torch.empty_like(q), torch.empty((Hq, T), device=DEV)
            sta.sta_paged_forward(q, o, cu, cache, max(new), cache.room, lse=lse)
            sta.sta_paged_weights(q, lse, w, cu, cache, max(new), cache.room, before=w, decay=0.5)
            outs.append((o, lse))
        assert all(same(a, b) for a, b in zip(*outs)), step
        for s, n in enumerate(own[now].used.tolist()):
            row = own[now].table[s].long()
            assert torch.equal(numbers[0][now][row].transpose(0, 1).flatten(1)[:, :n], numbers[1][now][s, :, :n]), (step, s)
    assert not torch.equal(numbers[1][0][0, :, :common * page], numbers[1][0][1, :, :common * page])       # of the shared pages, each its own


class Shared(Step):
    """The same step with the numbers by sequence."""

    def __init__(self, seed):
        super().__init__(seed)
        self.cache, self.into = (sta.StaPagedCache(c.k, c.v, c.table, c.used, shared=True) for c in (self.cache, self.into))
        self.w, self.to_w = (torch.zeros(c.weights_shape, device=DEV) for c in (self.cache, self.into))


def test_steps_replayed_from_a_graph():
    """Captured once and replayed with other lengths and rows, eager steps with the numbers by page and other work between: the same outputs, and the same numbers of the keys."""
    a, b = Shared(1), Step(1)
    for x in (a, b):
        x.fill(3)
        x.run()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        a.run()
    b.run()                                                     # capturing runs nothing: as many steps of either from here on
    graph.replay()
    for seed in (4, 9, 5, 2, 9):
        a.fill(seed)
        b.fill(seed)
        graph.replay()
        b.run()
        torch.cuda.synchronize()
        for x, y in zip((*a.pools, a.o, a.lse, a.into.k, a.into.v, a.into.used, a.kept), (*b.pools, b.o, b.lse, b.into.k, b.into.v, b.into.used, b.kept)):
            assert torch.equal(x, y), seed
        for c, x, y in ((a.cache, a.w, b.w), (a.into, a.to_w, b.to_w)):
            for s, n in enumerate(c.used.tolist()):
                assert torch.equal(x[s, :, :n], y[c.table[s].long()].transpose(0, 1).flatten(1)[:, :n]), (seed, s)
        assert bool(torch.isfinite(torch.randn((1 << 20,), device=DEV).sum()))
