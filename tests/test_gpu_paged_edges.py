"""The operators on a cache in pages at the edges of their arguments, on other streams and in graphs."""
import math

import pytest
import torch

import paper_2502_04507_amd as sta
from tests import layer_util as lu
from tests import paged_util as pu
from tests.paged_util import BF, DEV, Cache, forward, ints, packed, same, starts
from tests.test_gpu_packed import bounds, close, randn
from tests.test_gpu_paged_weights import allowed, gathered

pytestmark = pytest.mark.gpu
LOWEST = torch.finfo(BF).min

# single tokens whole and in parts; tiles by two groups, by four, in parts, and shared by four waves
SHAPES = [(4, 2, [1, 3], [40, 70]), (4, 2, [1, 2], [3000, 77]), (16, 8, [300] * 4, [300] * 4), (6, 3, [70, 45, 300], [70, 45, 300]), (8, 2, [100, 40], [4000, 300]),
          (32, 16, [520] * 9, [520] * 9)]


@pytest.mark.parametrize("kind", ["nan v", "inf v", "nan k", "inf k", "lowest k", "lowest v"])
@pytest.mark.parametrize("shape", SHAPES, ids=[str(i) for i in range(len(SHAPES))])
@pytest.mark.parametrize("page", [8, 5])
def test_what_is_no_number_or_the_lowest_one(shape, kind, page):
    """Keys that some rows see and others do not: the bits of sta_packed_forward on the same keys, which has its own tests."""
    Hq, Hkv, new, used = shape
    D = 64
    cache = Cache(Hkv, D, page, used, seed=4)
    value = {"nan": math.nan, "inf": math.inf, "lowest": LOWEST}[kind.split()[0]]
    for s in range(len(used)):
        j = max(0, used[s] - max(1, new[s] // 2))
        p, slot = cache.place(s, j)
        which = kind.endswith("k")
        (cache.k if which else cache.v)[s][j, 1, 3:5] = value
        cache.pool[0 if which else 1][p, slot, 1, 3:5] = value
    q = randn((sum(new), Hq, D), 3).to(DEV)
    for lse in (False, True):
        for a, b in zip(forward(q, cache, new, lse=lse), packed(q, cache, new, lse=lse)):
            if a is None:
                continue
            nan = torch.isnan(a)
            assert torch.equal(nan, torch.isnan(b)) and same(torch.where(nan, 0.0, a).to(a.dtype), torch.where(nan, 0.0, b).to(b.dtype))


@pytest.mark.parametrize("lse", [False, True])
@pytest.mark.parametrize("page,used", [(16, [16500, 40]), (3, [4500, 40]), (4, [8193, 8192])])
def test_walks_longer_than_the_places_that_are_kept(page, used, lse):
    """Tiles of 128 rows of 128 channels keep the places of 2048 groups of 4 rows, or rows where a page ends inside a group: walks that take several fillings, also a second time where V holds an
    infinity."""
    cache = Cache(8, 128, page, used, seed=4)
    new = [2400, 40]
    q = randn((2440, 32, 128), 6).to(DEV)
    for bad in (False, True):
        if bad:
            cache.v[0][used[0] - 100, 3, 7] = math.inf
            j, slot = cache.place(0, used[0] - 100)
            cache.pool[1][j, slot, 3, 7] = math.inf
        for got, want in zip(forward(q, cache, new, lse=lse), packed(q, cache, new, lse=lse)):
            assert got is None and want is None or same(got, want), bad
        assert not bad or bool(forward(q, cache, new)[0][2390, 12, 7] == math.inf)


def test_places_beyond_4_gb():
    """Pages 2.6 GB apart: the third lies beyond 32 bits of bytes, in either pool."""
    Hkv, Hq, D, page, stride = 2, 8, 128, 16, 1_300_000_000
    memory = torch.zeros(2 * stride + 2 * page * Hkv * D, dtype=BF, device=DEV)
    k, v = (torch.as_strided(memory, (3, page, Hkv, D), (stride, Hkv * D, D, 1), i * page * Hkv * D) for i in range(2))
    used, new = [40, 33], [3, 33]
    table = ints([[2, 0, 1], [1, 2, 0]])
    # page 2 is the first sequence's first and the second one's second: its rows are the same for both
    cache = sta.StaPagedCache(k, v, table, ints(used))
    x = randn((100, 2 * Hkv, D), 4).to(DEV)
    for i, p in enumerate((0, 1, 2)):
        k[p], v[p] = x[i * page:(i + 1) * page, :Hkv], x[i * page:(i + 1) * page, Hkv:]
    rows = [(2, 0, 1), (1, 2, 0)]
    K, V = ([torch.cat([t[p * page:(p + 1) * page] for p in r])[:n] for r, n in zip(rows, used)] for t in (x[:48, :Hkv].cpu(), x[:48, Hkv:].cpu()))
    q = randn((sum(new), Hq, D), 5)
    o, lse = torch.empty_like(q, device=DEV), torch.empty((Hq, sum(new)), device=DEV)
    cu = ints(starts(new))
    sta.sta_paged_forward(q.to(DEV), o, cu, cache, 33, 40, lse=lse)
    for s in range(2):
        a = slice(starts(new)[s], starts(new)[s + 1])
        want = lu.attention(q[a].double(), K[s].double(), V[s].double(), True, D ** -0.5)
        b_o, _, _ = bounds(q[a].double(), K[s].double(), V[s].double(), True, D ** -0.5, want[1])
        close(o[a], want[0], b_o, "sequence %d" % s)
    # weights of the first sequence alone, then its eviction within the same pool, and a row written into the far page
    one = sta.StaPagedCache(k, v, table[:1], ints(used[:1]))
    w = torch.zeros((3, Hkv, page), device=DEV)
    sta.sta_paged_weights(q[:3].to(DEV), lse[:, :3].contiguous(), w, ints([0, 3]), one, 3, 40)
    Q, z = q[:3].double(), lse[:, :3].cpu().double()
    want, off = pu.weights(Q, K[0].double(), z, True, D ** -0.5), allowed(Q, K[0].double(), z, True, D ** -0.5)
    got = w.cpu()[list(rows[0])].transpose(0, 1).flatten(1)[:, :40].double()
    assert bool(((got - want).abs() <= off + 2.0 ** -24 * want).all())
    near = [torch.zeros((2, page, Hkv, D), dtype=BF, device=DEV) for _ in range(2)]
    into, kept = sta.StaPagedCache(*near, ints([[1, 0]]), ints([0])), torch.zeros((1, Hkv, 20), dtype=torch.int32, device=DEV)
    sta.sta_paged_evict(one, w, into, None, kept, first=1, recent=2)
    for h in range(Hkv):
        stay = kept[0, h].cpu().long()
        assert stay.tolist() == pu.survivors(got[h].tolist(), 20, 1, 2)
        assert same(near[0][[1, 0]].flatten(0, 1)[:20, h].cpu(), K[0][stay, h]) and same(near[1][[1, 0]].flatten(0, 1)[:20, h].cpu(), V[0][stay, h])
    back = sta.StaPagedCache(k, v, ints([[2]]), ints([16]))
    sta.sta_paged_evict(into, torch.rand((2, Hkv, page), device=DEV), back, None, torch.zeros((1, Hkv, 16), dtype=torch.int32, device=DEV), recent=16)
    assert back.used.tolist() == [16] and same(k[2].cpu(), near[0][[1, 0]].flatten(0, 1)[4:20].cpu())
    sta.sta_paged_append(x[60:62, :Hkv], x[60:62, Hkv:], ints([0, 2]), back, 2)
    assert same(k[2, 14:], x[60:62, :Hkv]) and same(v[2, 14:], x[60:62, Hkv:])


def test_no_pages_no_keys_no_sequences():
    D, Hkv, Hq = 64, 2, 4
    k = torch.zeros((0, 16, Hkv, D), dtype=BF, device=DEV)
    for width in (0, 3):
        cache = sta.StaPagedCache(k, k, torch.zeros((2, width), dtype=torch.int32, device=DEV), ints([5, 9]))
        q = randn((60, Hq, D), 3).to(DEV)
        for new in ([2, 3], [20, 40]):
            o, lse = torch.full_like(q[:sum(new)], 7.0), torch.zeros((Hq, sum(new)), device=DEV)
            sta.sta_paged_forward(q[:sum(new)], o, ints(starts(new)), cache, max(new), 9, lse=lse)
            assert bool((o == 0).all()) and bool((lse == -math.inf).all())
        w = torch.zeros((0, Hkv, 16), device=DEV)
        sta.sta_paged_weights(q[:5], lse[:, :5].contiguous(), w, ints([0, 2, 5]), cache, 3, 9)
        sta.sta_paged_append(q[:5, :Hkv], q[:5, Hkv:], ints([0, 2, 5]), cache, 3)
        into = sta.StaPagedCache(torch.ones((1, 8, Hkv, D), dtype=BF, device=DEV), torch.ones((1, 8, Hkv, D), dtype=BF, device=DEV), ints([[0], [0]]), ints([4, 4]))
        kept = torch.zeros((2, Hkv, 8), dtype=torch.int32, device=DEV)
        sta.sta_paged_evict(cache, w, into, None, kept)
        assert bool((kept == -1).all()) and into.used.tolist() == [0, 0] and bool((into.k == 1).all())
    none = sta.StaPagedCache(k, k, torch.zeros((0, 4), dtype=torch.int32, device=DEV), torch.zeros(0, dtype=torch.int32, device=DEV))
    o = torch.full_like(q, 7.0)
    sta.sta_paged_forward(q, o, ints([0]), none, 5, 9)
    sta.sta_paged_append(q[:5, :Hkv], q[:5, Hkv:], ints([0]), none, 3)
    sta.sta_paged_evict(none, w, none, None, torch.zeros((0, Hkv, 0), dtype=torch.int32, device=DEV))
    assert bool((o == 7.0).all())


def test_evict_everything():
    cache = Cache(2, 64, 16, [100, 5], seed=6)
    w = torch.rand((cache.pages, 2, 16), device=DEV)
    k = torch.full((2, 16, 2, 64), 7.0, dtype=BF, device=DEV)
    into = sta.StaPagedCache(k, k.clone(), ints([[0], [1]]), ints([4, 4]))
    sta.sta_paged_evict(cache.sta, w, into, None, torch.zeros((2, 2, 0), dtype=torch.int32, device=DEV))
    assert into.used.tolist() == [0, 0] and bool((k == 7.0).all())


@pytest.mark.parametrize("Hq,Hkv,new,used", [(4, 2, [5, 3], [40, 300]), (4, 2, [60, 90], [70, 300])])
def test_weights_of_fewer_tokens_and_keys_than_there_are(Hq, Hkv, new, used):
    """max_q and max_k below the lengths: rows and keys beyond take no part, and nothing else changes."""
    D, max_q, max_k = 64, min(new) - 1, 64
    cache = Cache(Hkv, D, 16, used, seed=5)
    q = randn((sum(new), Hq, D), 3)
    _, lse = forward(q.to(DEV), cache, new, lse=True)
    w = torch.full((cache.pages, Hkv, 16), 7.0, device=DEV)
    sta.sta_paged_weights(q.to(DEV), lse, w, ints(starts(new)), cache.sta, max_q, max_k)
    cut = lse.clone()
    cu = starts(new)
    for s in range(2):
        cut[:, cu[s] + max_q:cu[s + 1]] = -math.inf             # rows that give nothing
    for s, n in enumerate(used):
        a = slice(cu[s], cu[s + 1])
        Q, K, z = q[a].double(), cache.k[s].double(), cut[:, a].cpu().double()
        want, off = pu.weights(Q, K, z, True, D ** -0.5), allowed(Q, K, z, True, D ** -0.5)
        got = gathered(cache, s, w)
        m = min(n, max_k)
        assert bool(((got - want).abs() <= off + 2.0 ** -24 * want)[:, :m].all()) and bool((got[:, m:] == 7.0).all())
    again = torch.zeros_like(w)                                 # and rows whose lse is -infinity give nothing, in the general way too
    sta.sta_paged_weights(q.to(DEV), cut, again, ints(cu), cache.sta, max(new), max(used))
    for s, n in enumerate(used):
        m = min(n, max_k)
        a, b = gathered(cache, s, again)[:, :m], gathered(cache, s, w)[:, :m]
        assert torch.allclose(a, b, rtol=1e-5, atol=1e-6)


@pytest.mark.parametrize("layout", ["heads", "wide"])
def test_queries_and_outputs_of_other_layouts(layout):
    Hq, Hkv, D, new, used = 6, 3, 64, [70, 2, 45], [170, 99, 45]
    cache = Cache(Hkv, D, 24, used, seed=5, layout="halves")
    q = randn((sum(new), Hq, D), 3)

    def dev(x):
        if layout == "heads":
            return x.transpose(0, 1).contiguous().to(DEV).transpose(0, 1)
        y = torch.full((x.shape[0], Hq + 2, D + 8), 7.0, dtype=BF, device=DEV)
        y[:, 1:-1, 8:] = x.to(DEV)
        return y[:, 1:-1, 8:]

    want, z = forward(q.to(DEV), cache, new, lse=True)
    got, z2 = forward(dev(q), cache, new, lse=True, o=dev(torch.zeros_like(q)))
    assert same(got, want) and same(z, z2)
    w = [torch.zeros((cache.pages, Hkv, 24), device=DEV) for _ in range(2)]
    for x, t in zip((q.to(DEV), dev(q)), w):
        sta.sta_paged_weights(x, z, t, ints(starts(new)), cache.sta, 70, 170)
    assert same(*w)


class Step:
    """One step of a program on buffers of its own: new rows, attention, weights, eviction into a second cache."""

    def __init__(self, seed):
        self.Hq, self.Hkv, self.D, self.page, self.S, self.T = 8, 2, 64, 16, 3, 80
        g = torch.Generator().manual_seed(seed)
        pages = 60
        self.pools = [torch.randn((pages, self.page, self.Hkv, self.D), generator=g).to(BF).to(DEV) for _ in range(2)]
        table = torch.randperm(pages, generator=g)[:self.S * 18].view(self.S, 18).to(torch.int32).to(DEV)
        self.cache = sta.StaPagedCache(*self.pools, table, ints([0, 0, 0]))
        self.into = sta.StaPagedCache(*[torch.zeros((12, self.page, self.Hkv, self.D), dtype=BF, device=DEV) for _ in range(2)],
                                      torch.arange(12, dtype=torch.int32, device=DEV).view(3, 4), ints([0, 0, 0]))
        self.x, self.q = torch.zeros((self.T, 2 * self.Hkv, self.D), dtype=BF, device=DEV), torch.zeros((self.T, self.Hq, self.D), dtype=BF, device=DEV)
        self.o, self.lse = torch.zeros_like(self.q), torch.zeros((self.Hq, self.T), device=DEV)
        self.cu = ints([0, 0, 0, 0])
        self.w, self.to_w = (torch.zeros((n, self.Hkv, self.page), device=DEV) for n in (pages, 12))
        self.kept = torch.zeros((self.S, self.Hkv, 64), dtype=torch.int32, device=DEV)
        n = sta.sta_paged_workspace_bytes(self.Hq, self.Hkv, self.D, self.S, self.T, 50, 288)
        self.ws = torch.empty(max(n, 16), dtype=torch.uint8, device=DEV)

    def fill(self, seed):
        g = torch.Generator().manual_seed(seed)
        new = [(seed * 7) % 50 + 1, seed % 3, (seed * 13) % 29]
        used = [max(n, (seed * 31 * (i + 1)) % 280) for i, n in enumerate(new)]
        self.x.copy_(torch.randn(self.x.shape, generator=g).to(BF))
        self.q.copy_(torch.randn(self.q.shape, generator=g).to(BF))
        self.cu.copy_(torch.tensor(starts(new), dtype=torch.int32))
        self.cache.used.copy_(torch.tensor(used, dtype=torch.int32))

    def run(self, stream=None):
        H = self.Hkv
        sta.sta_paged_append(self.x[:, :H], self.x[:, H:], self.cu, self.cache, 50, weights=self.w, stream=stream)
        sta.sta_paged_forward(self.q, self.o, self.cu, self.cache, 50, 288, lse=self.lse, workspace=self.ws, stream=stream)
        sta.sta_paged_weights(self.q, self.lse, self.w, self.cu, self.cache, 50, 288, before=self.w, decay=0.5, stream=stream)
        sta.sta_paged_evict(self.cache, self.w, self.into, self.to_w, self.kept, first=2, recent=10, stream=stream)

    def results(self):
        return [x.clone() for x in (*self.pools, self.o, self.lse, self.w, self.into.k, self.into.v, self.into.used, self.to_w, self.kept)]


def test_steps_replayed_from_a_graph():
    """Captured once, replayed with other lengths, rows and tables, eager steps and other work between: every replay against the same step made eagerly."""
    a, b = Step(1), Step(1)
    a.fill(3)
    b.fill(3)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):                               # a step before the capture, so that both have made as many
        a.run()
    torch.cuda.current_stream().wait_stream(side)
    b.run()
    graph = torch.cuda.CUDAGraph()
    a.fill(4)
    with torch.cuda.graph(graph):
        a.run()
    for seed in (4, 9, 5, 2, 9):
        a.fill(seed)
        b.fill(seed)
        graph.replay()
        b.run()
        torch.cuda.synchronize()
        for x, y in zip(a.results(), b.results()):
            assert torch.equal(x, y), seed
        junk = torch.randn((1 << 20,), device=DEV).sum()        # the program's own work between
        assert math.isfinite(float(junk))


def test_two_graphs_share_a_workspace():
    a, b, c = Step(1), Step(2), Step(2)
    b.ws = a.ws
    graphs = []
    for s in (a, b):
        s.fill(6)
        s.run()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            s.run()
        graphs.append(graph)
    c.fill(6)
    c.run()
    for seed in (7, 8, 6):
        for s in (a, b, c):
            s.fill(seed)
        graphs[0].replay()
        graphs[1].replay()
        c.run()
        torch.cuda.synchronize()
        for x, y in zip(b.results(), c.results()):
            assert torch.equal(x, y), seed


def test_on_another_stream():
    a, b = Step(5), Step(5)
    side = torch.cuda.Stream()
    for seed in (3, 4):
        a.fill(seed)
        b.fill(seed)
        torch.cuda.synchronize()
        if seed == 3:
            a.run(stream=side)
        else:
            with torch.cuda.stream(side):
                a.run()
        b.run()
        torch.cuda.synchronize()
        for x, y in zip(a.results(), b.results()):
            assert torch.equal(x, y)


@pytest.mark.parametrize("D", [64, 128])
def test_cut_chunks_replayed_with_other_lengths(D):
    """How long the parts of a walk are follows from the lengths on the device: a captured call replayed with others, parts of the replay before left in the workspace, against the same call made eagerly
    and the definition."""
    Hq, Hkv, page, S, T, max_k = 8, 2, 16, 3, 200, 12000
    g = torch.Generator().manual_seed(11)
    pages = S * (max_k // page)
    pool = [torch.randn((pages, page, Hkv, D), generator=g).to(BF).to(DEV) for _ in range(2)]
    table = torch.randperm(pages, generator=g).view(S, -1).to(torch.int32).to(DEV)
    cache, cu = sta.StaPagedCache(*pool, table, ints([0] * S)), ints([0] * (S + 1))
    q = randn((T, Hq, D), 12).to(DEV)
    n = sta.sta_paged_workspace_bytes(Hq, Hkv, D, S, T, T, max_k)
    assert n > 0
    ws = [torch.full((n,), 255, dtype=torch.uint8, device=DEV) for _ in range(2)]
    out = [(torch.full_like(q, 7.0), torch.full((Hq, T), 7.0, device=DEV)) for _ in range(2)]

    def call(i):
        sta.sta_paged_forward(q, out[i][0], cu, cache, T, max_k, lse=out[i][1], workspace=ws[i])

    call(0)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call(0)
    for new, used in (([100, 60, 40], [12000, 9000, 40]), ([200, 0, 0], [11999, 0, 5]), ([1, 1, 198], [12000, 1, 198]), ([0, 200, 0], [12000, 3000, 12000]), ([70, 70, 60], [100, 100, 60])):
        cu.copy_(torch.tensor(starts(new), dtype=torch.int32))
        cache.used.copy_(torch.tensor(used, dtype=torch.int32))
        graph.replay()
        call(1)
        torch.cuda.synchronize()
        for a, b in zip(*out):
            assert torch.equal(a, b), (new, used)
        at = starts(new)
        for s in range(S):
            rows, keys = slice(at[s], at[s + 1]), [x[table[s].long()].view(-1, Hkv, D)[:used[s]].cpu().double() for x in pool]
            Q = q[rows].cpu().double()
            want = lu.attention(Q, *keys, True, D ** -0.5)
            b_o, b_lse, _ = bounds(Q, *keys, True, D ** -0.5, want[1])
            close(out[0][0][rows], want[0], b_o, "sequence %d of %s" % (s, used))
            seen = want[1] > -math.inf
            z = out[0][1][:, rows].cpu().double()
            assert torch.equal(seen, z > -math.inf) and bool(((z - want[1])[seen].abs() <= b_lse[seen]).all()), (new, used)
