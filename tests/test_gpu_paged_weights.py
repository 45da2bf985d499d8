"""What keys of a cache in pages gather, the eviction by it, and a run of all operators on the cache, on the GPU, against plain implementations in 64 bits.

Allowed errors of a key's weight w_j = sum_i p_ij, p_ij = exp(scale q_i . k_j - lse_i) with lse_i the same fp32 numbers on both sides:
  scores     e_ij = (D + 4) 2^-24 of the sum of the absolute products (test_gpu_packed), times the scale, and the scale's own rounding and its product's with log2 e:
             3 2^-24 |s_ij|; lse_i's product with log2 e: 2 2^-24 |lse_i|; their difference, one rounding, 2^-24 (|s_ij| + |lse_i|); relative errors of p_ij all;
  exp2       2^-22 of p_ij;
  the sum    every addition 2^-24 of what is there so far, all terms positive: a stage's tree 3, sixteen stages, a sum every 512 rows, up to 4 groups and
             2 for the lanes: (25 + rows / 512) 2^-24 w_j; decay times what was there before and the sum, one rounding of the result."""
import math

import pytest
import torch

import paper_2502_04507_amd as sta
from tests import layer_util as lu
from tests import paged_util as pu
from tests.paged_util import BF, DEV, Cache, forward, ints, same, starts
from tests.test_gpu_packed import bounds, close, randn

pytestmark = pytest.mark.gpu
EPS = 2.0 ** -24


def allowed(q, k, lse, causal, scale):
    """[Hkv, lk]: what a key's weight may be off by, without what was there before."""
    lq, Hq, D = q.shape
    lk, Hkv = k.shape[0], k.shape[1]
    keep = lu.seen(lq, lk, causal)
    b = torch.zeros((Hkv, lk), dtype=torch.float64)
    for h in range(Hq):
        n = h // (Hq // Hkv)
        s, z = q[:, h] @ k[:, n].T * scale, lse[h][:, None]
        p = torch.where(keep & (z > -math.inf), torch.exp(s - z), 0.0)
        rel = (D + 4) * EPS * (q[:, h].abs() @ k[:, n].abs().T) * scale + 4 * EPS * s.abs() + 3 * EPS * torch.where(z == -math.inf, 0.0, z).abs() + 2.0 ** -22
        b[n] += (p * (rel + (25 + lq * Hq / Hkv / 512) * EPS)).sum(0)
    return b


def gathered(cache, s, w):
    """A sequence's numbers, [Hkv, used], of a device tensor [pages, Hkv, page]."""
    w = w.cpu()
    n = cache.used[s]
    return torch.cat([w[p] for p in cache.rows[s]] or [w[:0].reshape(cache.Hkv, 0)], 1)[:, :n].double()


def check_weights(cache, q, lse, new, causal=True, decay=1.0, before=True, scale=0.0, max_k=None):
    D, page, Hkv = cache.D, cache.page, cache.Hkv
    g = torch.Generator().manual_seed(17)
    old = torch.rand((cache.pages, Hkv, page), generator=g).to(DEV) if before else None
    if before and decay == 0.0:
        old.fill_(float("nan"))
    out = torch.full((cache.pages, Hkv, page), 7.0, device=DEV)
    runs = []
    for _ in range(2):
        sta.sta_paged_weights(q.to(DEV), lse, out, ints(starts(new)), cache.sta, max(new), max(cache.used) if max_k is None else max_k, before=old, decay=decay,
                              causal=causal, scale=scale)
        runs.append(out.clone())
    assert same(*runs)
    c = scale if scale > 0 else D ** -0.5
    cu, touched = starts(new), torch.zeros(out.shape, dtype=torch.bool)
    for s, n in enumerate(cache.used):
        a = slice(cu[s], cu[s + 1])
        Q, K, z = q[a].double(), cache.k[s].double(), lse[:, a].cpu().double()
        want, off = pu.weights(Q, K, z, causal, c), allowed(Q, K, z, causal, c)
        if before and decay != 0.0:
            want = want + decay * gathered(cache, s, old)
        got = gathered(cache, s, out)
        bound = off + EPS * (want.abs() + off)
        assert got.shape == want.shape and bool(((got - want).abs() <= bound).all()), (s, float(((got - want).abs() - bound).max()))
        for j, p in enumerate(cache.rows[s]):
            touched[p, :, :min(page, n - j * page)] = True
    assert bool((out.cpu()[~touched] == 7.0).all())             # other slots keep what they hold
    if before and decay != 0.0:                                 # in place
        sta.sta_paged_weights(q.to(DEV), lse, old, ints(starts(new)), cache.sta, max(new), max(cache.used) if max_k is None else max_k, before=old, decay=decay,
                              causal=causal, scale=scale)
        assert bool((old.cpu()[touched] == out.cpu()[touched]).all())
    return out


# Hq, Hkv, D, new, used, causal, page, decay: few rows; stages through LDS with four, two and one wave along the keys
WEIGHTS = [
    (4, 2, 128, [1, 1, 1], [77, 12, 1], True, 16, 1.0),
    (8, 1, 64, [2, 4, 1], [64, 4097, 300], True, 1, 0.0),
    (32, 8, 128, [1, 1], [5000, 31], True, 64, 0.96875),
    (8, 2, 128, [3, 8, 1], [300, 8, 129], True, 20, 1.0),
    (6, 3, 64, [70, 45, 300], [70, 145, 301], True, 3, 1.0),
    (15, 5, 64, [333, 1, 65], [1333, 97, 65], True, 256, 0.5),
    (8, 8, 128, [257, 33], [257, 1025], False, 40, 0.0),
    (16, 16, 64, [64] * 5, [1000] * 5, True, 24, 1.0),
    (16, 16, 128, [600, 40], [3000, 3001], True, 32, 1.0),
    (40, 8, 128, [40, 100], [6000, 5100], True, 16, -1.5),
    (2, 1, 64, [5000], [5000], True, 128, 1.0),
]


@pytest.mark.parametrize("case", [(16, 16, 64, [700, 30], [3000, 1500], True, 16, 0.5), (16, 16, 64, [600, 513, 0], [5000, 4000, 200], True, 1, 1.0),
                                  (24, 8, 64, [300, 250], [7000, 6500], False, 20, 1.0), (24, 8, 64, [300, 1], [301, 7000], True, 64, 1.0)], ids=["0", "1", "2", "3"])
def test_weights_of_many_rows_of_64_channels(case):
    """More than 512 rows of a key head: two waves along the keys by two groups with stages of 64 rows."""
    Hq, Hkv, D, new, used, causal, page, decay = case
    cache = Cache(Hkv, D, page, used, seed=15)
    q = randn((sum(new), Hq, D), 13)
    _, lse = forward(q.to(DEV), cache, new, causal=causal, lse=True)
    check_weights(cache, q, lse, new, causal, decay)


@pytest.mark.parametrize("case", [(16, 16, 128, [100, 40], [9500, 4000], True, 16, 0.5), (16, 16, 128, [100, 40, 0, 60], [8300, 4000, 129, 1], False, 5, 1.0),
                                  (15, 5, 128, [50, 60, 1], [14000, 12900, 300], True, 64, 1.0), (15, 5, 128, [40, 1, 39], [14000, 12900, 12345], True, 1, 0.0)], ids=["0", "1", "2", "3"])
def test_weights_of_rounds_of_tiles(case):
    """Tiles of 256 keys of 128 channels, the last few of the many in halves, of which one may have no key."""
    Hq, Hkv, D, new, used, causal, page, decay = case
    cache = Cache(Hkv, D, page, used, seed=25)
    q = randn((sum(new), Hq, D), 23)
    _, lse = forward(q.to(DEV), cache, new, causal=causal, lse=True)
    check_weights(cache, q, lse, new, causal, decay)


@pytest.mark.parametrize("case", WEIGHTS, ids=[str(i) for i in range(len(WEIGHTS))])
def test_weights(case):
    Hq, Hkv, D, new, used, causal, page, decay = case
    cache = Cache(Hkv, D, page, used, seed=5, layout=("tokens", "heads", "halves")[len(used) % 3])
    q = randn((sum(new), Hq, D), 3)
    print(case, flush=True)
    _, lse = forward(q.to(DEV), cache, new, causal=causal, lse=True)
    check_weights(cache, q, lse, new, causal, decay)
    check_weights(cache, q, lse, new, causal, decay, before=False)
    out = check_weights(cache, q, lse, new, causal, 0.0, before=False, scale=0.0)
    for s, n in enumerate(new):                                 # every row that sees a key gives 1 in all
        rows = (torch.minimum(torch.tensor(used[s]), torch.tensor(n)) if causal else torch.tensor(n)).item() * Hq // Hkv
        assert gathered(cache, s, out).sum(1) == pytest.approx(rows, rel=1e-4)


@pytest.mark.parametrize("new,given", [([3, 1, 2], [0, 2, 96]), ([60, 90, 64], [0, 2, 96]), ([5, 64, 90], [3, 40, 96])])
def test_weights_of_rows_without_keys_and_lengths_beyond_the_table(new, given):
    cache = Cache(2, 64, 16, given, seed=11, room=6)
    cache.lengths.copy_(ints([x if x < 96 else 5000 for x in given]))
    q = randn((sum(new), 4, 64), 4)
    _, lse = forward(q.to(DEV), cache, new, lse=True, max_k=5000)
    check_weights(cache, q, lse, new, max_k=5000)


def test_no_new_tokens_leave_the_decay():
    cache = Cache(2, 128, 16, [40, 33], seed=11)
    w = torch.full((cache.pages, 2, 16), 3.0, device=DEV)
    q, lse = torch.zeros((0, 4, 128), dtype=BF, device=DEV), torch.zeros((4, 0), device=DEV)
    sta.sta_paged_weights(q, lse, w, ints([0, 0, 0]), cache.sta, 0, 40, before=w, decay=0.5)
    for s in range(2):
        assert bool((gathered(cache, s, w) == 1.5).all())
    assert int((w == 3.0).sum()) == w.numel() - 2 * 73


@pytest.mark.parametrize("new,rows", [([2, 1], 0), ([70, 45], 40)])
@pytest.mark.parametrize("which", ["q", "k", "lse"])
def test_nan_stays_with_the_rows_and_keys_that_meet(which, new, rows):
    Hq, Hkv, D, used = 4, 2, 64, [130, 90]
    cache = Cache(Hkv, D, 16, used, seed=5)
    q = randn((sum(new), Hq, D), 3)
    _, lse = forward(q.to(DEV), cache, new, lse=True)
    want = torch.zeros((cache.pages, Hkv, 16), device=DEV)
    args = (ints(starts(new)), cache.sta, max(new), max(used))
    sta.sta_paged_weights(q.to(DEV), lse, want, *args)
    token = rows                                                # of sequence 0
    sees = used[0] - new[0] + token + 1
    if which == "q":
        q[token, 1, 5] = float("nan")                           # head 1: of key head 0
    elif which == "lse":
        lse[1, token] = float("nan")
    else:
        p, slot = cache.place(0, 7)
        cache.pool[0][p, slot, 0, 3] = float("nan")
    got = torch.zeros_like(want)
    sta.sta_paged_weights(q.to(DEV), lse, got, *args)
    nan = torch.zeros((Hkv, used[0]), dtype=torch.bool)
    if which == "k":
        nan[0, 7] = True
    else:
        nan[0, :sees] = True
    a, b = gathered(cache, 0, got), gathered(cache, 0, want)
    assert torch.equal(torch.isnan(a), nan) and torch.equal(a[~nan], b[~nan])
    assert torch.equal(gathered(cache, 1, got), gathered(cache, 1, want))


def test_a_window_of_the_last_rows():
    """The last 32 of a prompt's rows alone: their part of q and lse, given as strided views."""
    cache = Cache(4, 128, 64, [900], seed=5)
    q = randn((900, 8, 128), 3)
    _, lse = forward(q.to(DEV), cache, [900], lse=True)
    check_weights(cache, q[-32:], lse[:, -32:].contiguous(), [32])


# ---- eviction: moves and comparisons, so every bit is known
def evict(cache, w, keep, first, recent, page=None, to_weights=True, same_pool=False):
    """Returns what is in the new pages: lists of k, v, weights and kept indices."""
    S, Hkv, D = len(cache.used), cache.Hkv, cache.D
    page = page or cache.page
    need = max(1, -(-keep // page))
    if same_pool:                                               # pages behind those of the cache
        k, v = (torch.cat((x, torch.zeros((S * need + 2, page, Hkv, D), dtype=BF, device=DEV))) for x in cache.pool)
        w = torch.cat((w, torch.full((S * need + 2, Hkv, page), 7.0, device=DEV)))
        cache.sta = sta.StaPagedCache(k, v, cache.table, cache.lengths)
        to_w, base = w, cache.pages
    else:
        k, v = (torch.full((S * need + 2, Hkv, page, D), 7.0, dtype=BF, device=DEV).transpose(1, 2) for _ in range(2))
        to_w, base = torch.full((S * need + 2, Hkv, page), 7.0, device=DEV), 0
    order = torch.randperm(S * need + 2, generator=torch.Generator().manual_seed(3))[:S * need].view(S, need).to(torch.int32) + base
    to_used = torch.full((S,), -3, dtype=torch.int32, device=DEV)
    into = sta.StaPagedCache(k, v, order.to(DEV), to_used)
    kept = torch.full((S, Hkv, keep), -9, dtype=torch.int32, device=DEV)
    for _ in range(2):
        assert sta.sta_paged_evict(cache.sta, w, into, to_w if to_weights else None, kept, first=first, recent=recent) is into
    out_k, out_v, out_w = [], [], []
    for s in range(S):
        row = order[s].long().to(DEV)
        out_k.append(k[row].flatten(0, 1)[:keep].cpu())
        out_v.append(v[row].flatten(0, 1)[:keep].cpu())
        out_w.append(to_w[row].transpose(1, 2).flatten(0, 1)[:keep].cpu())
    unused = torch.ones(k.shape[0], dtype=torch.bool)
    unused[order.flatten().long()] = False
    unused[:base] = False
    filler = 0.0 if same_pool else 7.0
    assert bool((k[unused.to(DEV)] == filler).all()) and bool((to_w[unused.to(DEV)] == 7.0).all())
    return out_k, out_v, out_w, kept.cpu(), to_used.cpu()


def check_evict(cache, w, keep, first, recent, **kw):
    k, v, out_w, kept, to_used = evict(cache, w, keep, first, recent, **kw)
    for s, n in enumerate(cache.used):
        stay = min(n, keep)
        assert int(to_used[s]) == stay
        given = gathered(cache, s, w)
        for h in range(cache.Hkv):
            order = [math.inf if math.isnan(x) else x for x in given[h].tolist()]
            nans = [j for j, x in enumerate(given[h].tolist()) if math.isnan(x)]
            if nans:                                            # above infinity: told apart by their rank
                order = [2.0 if j in set(nans) else 1.0 if x == math.inf else math.atan(x) / 2 for j, x in enumerate(order)]
            want = pu.survivors(order, keep, first, recent)
            assert kept[s, h, :stay].tolist() == want and bool((kept[s, h, stay:] == -1).all()), (s, h)
            assert same(k[s][:stay, h], cache.k[s][want, h]) and same(v[s][:stay, h], cache.v[s][want, h]), (s, h)
            if kw.get("to_weights", True):
                assert torch.equal(out_w[s][:stay, h].double().nan_to_num(9e9), given[h][want].nan_to_num(9e9)), (s, h)


@pytest.mark.parametrize("kw", [dict(), dict(page=5), dict(same_pool=True), dict(to_weights=False)])
@pytest.mark.parametrize("Hkv,D,page,used,keep,first,recent", [
    (2, 128, 16, [300, 128, 127, 129, 0, 1], 128, 4, 32), (5, 64, 7, [100, 2000], 33, 0, 0), (1, 64, 64, [70], 64, 64, 0), (3, 128, 1, [90, 10], 20, 0, 20),
    (2, 64, 16, [500], 1, 0, 0), (2, 64, 16, [500, 3], 1, 1, 0), (2, 128, 100, [5000, 1100], 1024, 3, 61), (1, 128, 16, [40], 39, 1, 1),
])
def test_evict(Hkv, D, page, used, keep, first, recent, kw):
    cache = Cache(Hkv, D, page, used, seed=6, layout=("tokens", "heads", "halves")[Hkv % 3] if not kw.get("same_pool") else "tokens")
    g = torch.Generator().manual_seed(8)
    w = torch.randn((cache.pages, Hkv, page), generator=g).exp() * (torch.rand((cache.pages, Hkv, page), generator=g) < 0.8)
    check_evict(cache, w.to(DEV), keep, first, recent, **kw)


@pytest.mark.parametrize("kind", ["equal", "two", "signed zeros", "negative", "infinities", "nan", "near", "denormal"])
def test_evict_by_weights_that_are_hard_to_tell_apart(kind):
    Hkv, D, page, used = 2, 64, 16, [3000, 257, 300]
    cache = Cache(Hkv, D, page, used, seed=6)
    g = torch.Generator().manual_seed(9)
    shape = (cache.pages, Hkv, page)
    u = torch.rand(shape, generator=g)
    w = {"equal": torch.ones(shape), "two": (u < 0.1).float(), "signed zeros": torch.where(u < 0.5, 0.0, -0.0), "negative": torch.randn(shape, generator=g),
         "infinities": torch.where(u < 0.1, math.inf, torch.where(u < 0.2, -math.inf, torch.randn(shape, generator=g))), "nan": torch.where(u < 0.05, math.nan, torch.where(u < 0.1, math.inf, u)),
         "near": 1.0 + torch.randint(0, 700, shape, generator=g) * 2.0 ** -23, "denormal": torch.randint(0, 100, shape, generator=g) * 2.0 ** -149}[kind]
    check_evict(cache, w.to(DEV), 256, 2, 30)


def test_evict_more_keys_than_a_workgroup_has_threads_many_times():
    Hkv, D, page, used = 1, 64, 64, [40000, 32769]
    cache = Cache(Hkv, D, page, used, seed=6)
    w = torch.randn((cache.pages, Hkv, page), generator=torch.Generator().manual_seed(8)).exp()
    check_evict(cache, w.to(DEV), 4097, 4, 64)


def test_evict_writes_nothing_for_entries_that_are_no_pages():
    cache = Cache(2, 64, 16, [100, 50], seed=6)
    w = torch.rand((cache.pages, 2, 16), device=DEV)
    k, v = (torch.full((4, 16, 2, 64), 7.0, dtype=BF, device=DEV) for _ in range(2))
    to_w = torch.full((4, 2, 16), 7.0, device=DEV)
    into = sta.StaPagedCache(k, v, ints([[0, -1], [1 << 30, 2]]), ints([0, 0]))
    kept = torch.zeros((2, 2, 32), dtype=torch.int32, device=DEV)
    sta.sta_paged_evict(cache.sta, w, into, to_w, kept)
    assert bool((k[[1, 3]] == 7.0).all()) and bool((v[[1, 3]] == 7.0).all()) and bool((to_w[[1, 3]] == 7.0).all())
    for s, page, at in ((0, 0, 0), (1, 2, 16)):
        for h in range(2):
            assert same(k[page, :, h].cpu(), cache.k[s][kept[s, h, at:at + 16].cpu().long(), h])
    assert into.used.tolist() == [32, 32]


# ---- all of them, as a program uses them
def test_a_conversation():
    """Prompts into the cache and through it, what their last rows look at, eviction to a budget, then tokens one by one whose weights are added up, and another
    eviction: every step's output against the definition on the keys that are there by then, a list of rows for every key head."""
    Hq, Hkv, D, page, keep, S = 8, 2, 128, 16, 96, 3
    lengths, pages = [300, 41, 150], 64
    g = torch.Generator().manual_seed(21)

    def randn(*shape):
        return torch.randn(shape, generator=g).to(BF)

    pools = [torch.full((pages, page, Hkv, D), float("nan"), dtype=BF, device=DEV) for _ in range(4)]
    weights = [torch.full((pages, Hkv, page), float("nan"), device=DEV) for _ in range(2)]
    table = torch.randperm(pages, generator=g)[:3 * 20].view(S, 20).to(torch.int32).to(DEV)
    caches = [sta.StaPagedCache(pools[2 * i], pools[2 * i + 1], table, torch.zeros(S, dtype=torch.int32, device=DEV)) for i in range(2)]
    kept = torch.empty((S, Hkv, keep), dtype=torch.int32, device=DEV)
    have = [[(torch.zeros((0, D), dtype=BF),) * 2 for _ in range(Hkv)] for _ in range(S)]        # the model: rows of k and v of every head
    now = 0

    def step(new, window):
        q, k, v = randn(sum(new), Hq, D), randn(sum(new), Hkv, D), randn(sum(new), Hkv, D)
        cache, w = caches[now], weights[now]
        cu, longest = ints(starts(new)), int(cache.used.max()) + max(new)
        cache.used.add_(ints(new))
        sta.sta_paged_append(k.to(DEV), v.to(DEV), cu, cache, max(new), weights=w)
        qd, o, lse = q.to(DEV), torch.empty_like(q, device=DEV), torch.empty((Hq, sum(new)), device=DEV)
        n = sta.sta_paged_workspace_bytes(Hq, Hkv, D, S, sum(new), max(new), longest)
        sta.sta_paged_forward(qd, o, cu, cache, max(new), longest, lse=lse, workspace=torch.empty(max(n, 16), dtype=torch.uint8, device=DEV))
        last = [min(window, n) for n in new]
        rows = torch.cat([torch.arange(c + n - m, c + n) for c, n, m in zip(starts(new), new, last)]).to(DEV)
        sta.sta_paged_weights(qd[rows], lse[:, rows].contiguous(), w, ints(starts(last)), cache, max(last), longest, before=w)
        return q, k, v, o, lse, last

    def check(new, q, k, v, o, lse, last, model_weights):
        cu = starts(new)
        for s, n in enumerate(new):
            a = slice(cu[s], cu[s + 1])
            for h in range(Hkv):
                have[s][h] = (torch.cat((have[s][h][0], k[a, h])), torch.cat((have[s][h][1], v[a, h])))
            K, V = (torch.stack([have[s][h][i] for h in range(Hkv)], 1).double() for i in range(2))
            Q = q[a].double()
            want = lu.attention(Q, K, V, True, D ** -0.5)
            b_o, _, _ = bounds(Q, K, V, True, D ** -0.5, want[1])
            close(o[a], want[0], b_o, "sequence %d" % s)
            z = lse[:, a].cpu().double()[:, n - last[s]:]
            add, off = pu.weights(Q[n - last[s]:], K, z, True, D ** -0.5), allowed(Q[n - last[s]:], K, z, True, D ** -0.5)
            old, old_off = model_weights[s]
            pad = torch.zeros((Hkv, K.shape[0] - old.shape[1]), dtype=torch.float64)
            total, slack = torch.cat((old, pad), 1) + add, torch.cat((old_off, pad), 1) + off
            model_weights[s] = (total, slack + EPS * (total + slack))

    model = [(torch.zeros((Hkv, 0), dtype=torch.float64),) * 2 for _ in range(S)]

    def evict_both():
        nonlocal now
        w = weights[now].cpu().double()
        sta.sta_paged_evict(caches[now], weights[now], caches[1 - now], weights[1 - now], kept, first=2, recent=16)
        for s in range(S):
            K = have[s][0][0].shape[0]
            row = table[s].long().cpu()
            there = w[row].transpose(0, 1).flatten(1)[:, :K]                        # what the device holds, near the model, decides
            assert bool(((there - model[s][0]).abs() <= model[s][1]).all()), s
            keeps = [pu.survivors(there[h].tolist(), keep, 2, 16) for h in range(Hkv)]
            for h in range(Hkv):
                assert kept[s, h, :len(keeps[h])].tolist() == keeps[h], (s, h)
                have[s][h] = tuple(x[keeps[h]] for x in have[s][h])
            model[s] = tuple(torch.stack([x[h][keeps[h]] for h in range(Hkv)]) for x in model[s])
        now = 1 - now

    check(lengths, *step(lengths, 32), model)
    evict_both()
    assert caches[now].used.tolist() == [96, 41, 96]
    for i in range(20):
        new = [1, 1, 1] if i != 7 else [1, 3, 0]
        check(new, *step(new, 4), model)
    evict_both()
    check([1, 1, 1], *step([1, 1, 1], 4), model)
