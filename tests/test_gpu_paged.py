"""Attention over a cache in pages and the rows written into it, on the GPU: against the definition in 64 bits with the errors that test_gpu_packed derives, and against
sta_packed_forward on the same keys side by side, whose bits it has."""
import math

import pytest
import torch

import paper_2502_04507_amd as sta
from tests import layer_util as lu
from tests.paged_util import BF, DEV, Cache, forward, ints, packed, same, starts
from tests.test_gpu_packed import bounds, close, randn

pytestmark = pytest.mark.gpu

# Hq, Hkv, D, new, used, causal, page: single tokens and few rows, whole and in parts of the keys; tiles by one, two and four groups, whole and in parts
CASES = [
    (4, 2, 128, [1, 1, 1], [77, 12, 1], True, 16),
    (8, 8, 64, [1, 3, 2], [1, 33, 100], True, 8),
    (8, 1, 128, [2, 4, 1], [64, 4097, 300], True, 1),
    (32, 8, 128, [1, 1], [5000, 31], True, 64),
    (5, 5, 64, [7, 16, 1], [3000, 16, 45], False, 20),
    (6, 3, 128, [33, 45, 1], [33, 145, 2], True, 24),
    (6, 3, 64, [70, 45, 300], [70, 145, 301], True, 3),
    (16, 8, 128, [300] * 4, [300, 310, 555, 999], True, 32),
    (15, 5, 64, [333, 1, 65], [1333, 97, 65], True, 256),
    (8, 2, 128, [100, 40], [4000, 300], True, 16),
    (8, 2, 64, [100, 40], [9000, 41], True, 7),
    (32, 16, 64, [520] * 9, [520] * 9, True, 100),
    (16, 16, 128, [257, 200], [257, 1025], False, 40),
    (24, 24, 128, [260] * 3, [260, 300, 420], True, 6),
]


@pytest.mark.parametrize("lse", [False, True])
@pytest.mark.parametrize("case", CASES, ids=[str(i) for i in range(len(CASES))])
def test_the_same_as_keys_side_by_side_and_the_definition(case, lse):
    Hq, Hkv, D, new, used, causal, page = case
    cache = Cache(Hkv, D, page, used, seed=5, layout=("tokens", "heads", "halves")[len(used) % 3])
    q = randn((sum(new), Hq, D), 3)
    qd = q.to(DEV)
    for workspace in (True, False):
        print(case, lse, workspace, flush=True)
        o, z = forward(qd, cache, new, causal=causal, lse=lse, workspace=workspace)
        o2, z2 = packed(qd, cache, new, causal=causal, lse=lse, workspace=workspace)
        assert same(o, o2) and (not lse or same(z, z2))
    cu = starts(new)
    for s in range(len(new)):
        a = slice(cu[s], cu[s] + new[s])
        Q, K, V = q[a].double(), cache.k[s].double(), cache.v[s].double()
        want = lu.attention(Q, K, V, causal, D ** -0.5)
        b_o, b_lse, _ = bounds(Q, K, V, causal, D ** -0.5, want[1])
        close(o[a], want[0], b_o, "sequence %d" % s)
        if lse:
            assert bool(((z[:, a].cpu().double() - want[1]).abs() <= b_lse).all()), s


def test_walks_of_uneven_lengths():
    """Tiles by four groups where those of packed sequences are by two: other orders of sums, so against the definition alone, and the same whatever the pages are."""
    Hq, Hkv, D, new, used = 24, 24, 64, [300, 1, 1, 200], [3100, 3000, 50, 200]
    cache = Cache(Hkv, D, 24, used, seed=5)
    q = randn((sum(new), Hq, D), 3)
    o, z = forward(q.to(DEV), cache, new, lse=True)
    other = Cache(Hkv, D, 64, used, seed=6, layout="heads", keys=(cache.k, cache.v))
    for a, b in zip((o, z), forward(q.to(DEV), other, new, lse=True)):
        assert same(a, b)
    cu = starts(new)
    for s in range(len(new)):
        a = slice(cu[s], cu[s] + new[s])
        Q, K, V = q[a].double(), cache.k[s].double(), cache.v[s].double()
        want = lu.attention(Q, K, V, True, D ** -0.5)
        b_o, b_lse, _ = bounds(Q, K, V, True, D ** -0.5, want[1])
        close(o[a], want[0], b_o, "sequence %d" % s)
        assert bool(((z[:, a].cpu().double() - want[1]).abs() <= b_lse).all()), s


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("new,used", [([100, 80], [9000, 8200]), ([200, 10, 1], [9001, 300, 9000]), ([130, 130, 130], [8200, 130, 100]), ([9] * 66, [9000] + [20] * 65)])
def test_chunks_that_are_cut_along_the_keys(new, used, D):
    """Tiles of 128 rows in parts, of alike and of uneven lengths, more than 64 of them, sequences with fewer keys than a part and with fewer keys than rows among them."""
    Hq, Hkv = 8, 2
    assert sta.sta_paged_workspace_bytes(Hq, Hkv, D, len(new), sum(new), max(new), max(used)) > 0
    cache = Cache(Hkv, D, 16, used, seed=7)
    q = randn((sum(new), Hq, D), 8)
    o, z = forward(q.to(DEV), cache, new, lse=True)
    other = Cache(Hkv, D, 3, used, seed=9, layout="heads", keys=(cache.k, cache.v))
    for a, b in zip((o, z), forward(q.to(DEV), other, new, lse=True)):
        assert same(a, b)
    cu = starts(new)
    for s in range(len(new)):
        a = slice(cu[s], cu[s] + new[s])
        Q, K, V = q[a].double(), cache.k[s].double(), cache.v[s].double()
        want = lu.attention(Q, K, V, True, D ** -0.5)
        b_o, b_lse, _ = bounds(Q, K, V, True, D ** -0.5, want[1])
        close(o[a], want[0], b_o, "sequence %d" % s)
        seen = want[1] > -math.inf
        assert torch.equal(seen, z[:, a].cpu() > -math.inf)
        assert bool(((z[:, a].cpu().double() - want[1])[seen].abs() <= b_lse[seen]).all()), s


@pytest.mark.parametrize("layout", ["tokens", "heads", "halves"])
@pytest.mark.parametrize("page", [1, 4, 5, 8, 32, 33, 128])
@pytest.mark.parametrize("D", [64, 128])
def test_pages_of_any_size_and_layout(D, page, layout):
    for Hq, Hkv, new, used in ((8, 2, [1, 2, 1], [31, 200, 32]), (6, 3, [40, 90], [140, 131])):
        cache = Cache(Hkv, D, page, used, seed=7, layout=layout)
        q = randn((sum(new), Hq, D), 4).to(DEV)
        print(D, page, layout, new, flush=True)
        for got, want in zip(forward(q, cache, new, lse=True), packed(q, cache, new, lse=True)):
            assert same(got, want)


@pytest.mark.parametrize("new", [[1, 2], [60, 90]])
def test_sequences_share_pages(new):
    """A common beginning: the same pages in both rows of the table."""
    D, Hkv, page = 128, 2, 16
    cache = Cache(Hkv, D, page, [200, 150], seed=9)
    shared = 5
    cache.table[1, :shared] = cache.table[0, :shared]
    cache.k[1][:shared * page], cache.v[1][:shared * page] = cache.k[0][:shared * page], cache.v[0][:shared * page]
    q = randn((sum(new), 4, D), 4).to(DEV)
    for got, want in zip(forward(q, cache, new, lse=True), packed(q, cache, new, lse=True)):
        assert same(got, want)


@pytest.mark.parametrize("new", [[3, 1, 2, 5], [60, 90, 64, 40]])
def test_lengths_of_none_below_the_new_tokens_and_beyond_the_table(new):
    """Used lengths of 0 and below, fewer keys than tokens (rows that see none), and lengths that the table has no places for, which are cut."""
    D, Hkv, Hq, page = 64, 2, 4, 16
    given = [0, 2, 64, 96]
    cache = Cache(Hkv, D, page, given, seed=11, room=6)
    cache.lengths.copy_(ints([-7, 2, 64, 5000]))
    q = randn((sum(new), Hq, D), 4)
    o, lse = forward(q.to(DEV), cache, new, lse=True, max_k=5000)
    cu = starts(new)
    for s, n in enumerate(new):
        a = slice(cu[s], cu[s + 1])
        Q, K, V = q[a].double(), cache.k[s].double(), cache.v[s].double()
        want = lu.attention(Q, K, V, True, D ** -0.5)
        b_o, b_lse, _ = bounds(Q, K, V, True, D ** -0.5, want[1])
        close(o[a], want[0], b_o, "sequence %d" % s, norm=False)
        got = lse[:, a].cpu().double()
        seen = ~torch.isinf(want[1])
        assert torch.equal(got == -math.inf, ~seen) and bool(((got - want[1]).abs()[seen] <= b_lse[seen]).all()), s


@pytest.mark.parametrize("new", [[1, 1], [70, 40]])
def test_entries_that_are_no_pages_are_read_inside_the_pool(new):
    D, Hkv, Hq, page = 128, 2, 4, 16
    cache = Cache(Hkv, D, page, [100, 70], seed=13)
    for x in cache.pool:                        # every page holds numbers, so whatever is read gives numbers
        x.copy_(randn(x.shape, 5).to(DEV))
    q = randn((sum(new), Hq, D), 4).to(DEV)
    want, _ = forward(q, cache, new)
    cache.table[0, :3] = ints([-1, 1 << 30, -(1 << 31)])
    got, _ = forward(q, cache, new)
    assert bool(torch.isfinite(got).all())
    assert same(got[new[0]:], want[new[0]:]) and not same(got[:new[0]], want[:new[0]])


def test_tokens_of_no_sequence_keep_what_o_holds():
    D, Hkv, Hq = 64, 2, 4
    cache = Cache(Hkv, D, 16, [100, 70], seed=13)
    q = randn((10, Hq, D), 4).to(DEV)
    o, lse = torch.full_like(q, 7.0), torch.full((Hq, 10), 7.0, device=DEV)
    sta.sta_paged_forward(q, o, ints([2, 5, 7]), cache.sta, 3, 100, lse=lse)
    rest = torch.tensor([0, 1, 7, 8, 9], device=DEV)
    assert bool((o[rest] == 7.0).all()) and bool((lse[:, rest] == 7.0).all()) and not bool((o[2:7] == 7.0).all(-1).any())


# ---- new rows into their pages: moved, or rounded once to the nearest, so every bit is known
@pytest.mark.parametrize("dtype", [BF, torch.float32])
@pytest.mark.parametrize("Hkv,D,page,new,used,layout", [
    (1, 64, 16, [1], [1], "tokens"), (8, 128, 16, [1] * 5, [1, 16, 17, 32, 100], "heads"), (5, 64, 1, [3, 0, 7], [10, 4, 7], "halves"),
    (3, 128, 24, [333, 1, 25], [400, 24, 25], "tokens"), (2, 64, 100, [2, 1, 250], [2, 0, 199], "heads"), (40, 128, 7, [9, 30], [10, 45], "tokens"),
])
def test_append(Hkv, D, page, new, used, layout, dtype):
    """used below new: the first of the new tokens have no key."""
    cache = Cache(Hkv, D, page, used, seed=3, layout=layout)
    x = randn((sum(new), 2 * Hkv + 1, D + 8), 4).to(dtype) * (1 + 2.0 ** -9)           # float32: halfway and other places between bf16 numbers
    x = x.to(dtype)
    k, v = x[:, :Hkv, 8:], x[:, Hkv:2 * Hkv, 8:]
    weights = torch.full((cache.pages, Hkv, page), 3.0, device=DEV)
    want_k, want_v, want_w = (t.cpu().clone() for t in (*cache.pool, weights))
    cu = starts(new)
    for s, n in enumerate(new):
        for i in range(n):
            key = used[s] - n + i
            if key < 0:
                continue
            p, slot = cache.place(s, key)
            want_k[p, slot], want_v[p, slot], want_w[p, :, slot] = k[cu[s] + i].to(BF), v[cu[s] + i].to(BF), 0.0
    xd = x.to(DEV)
    for w in (weights, None):
        sta.sta_paged_append(xd[:, :Hkv, 8:], xd[:, Hkv:2 * Hkv, 8:], ints(cu), cache.sta, max(new), weights=w)
        assert same(cache.pool[0].cpu(), want_k) and same(cache.pool[1].cpu(), want_v) and same(weights.cpu(), want_w)


def test_append_writes_nothing_outside():
    """Tokens beyond max_new, keys beyond the table, entries that are no pages, sequences whose bounds leave the tokens."""
    Hkv, D, page = 2, 64, 8
    cache = Cache(Hkv, D, page, [24, 16, 8, 8], seed=3, room=3)
    cache.lengths.copy_(ints([40, 16, -5, 8]))
    cache.table[1, 0] = -1
    cache.table[1, 1] = cache.pages
    x = randn((30, Hkv, D), 4).to(DEV)
    want = [t.clone() for t in cache.pool]
    cu = ints([0, 20, 25, 28, 1000])                    # the last sequence's end is behind the tokens: it has two
    sta.sta_paged_append(x, x, cu, cache.sta, 6)
    # sequence 0: 20 tokens become keys 20 .. 39, six of them looked at, four with a place; 1 has no pages, 2 no keys; 3: two tokens become keys 6 and 7
    for s, n, key0, count in ((0, 0, 20, 4), (3, 28, 6, 2)):
        for i in range(count):
            p, slot = cache.place(s, key0 + i)
            for t in want:
                t[p, slot] = x[n + i]
    assert all(same(a, b) for a, b in zip(cache.pool, want))


def test_append_many_short_and_one_long_sequence():
    """More tokens of one sequence than its workgroups take at once."""
    Hkv, D, page = 2, 64, 16
    new = [1] * 200 + [5000] + [2] * 100
    cache = Cache(Hkv, D, page, new, seed=3)
    x = randn((sum(new), 2 * Hkv, D), 4)
    xd = x.to(DEV)
    sta.sta_paged_append(xd[:, :Hkv], xd[:, Hkv:], ints(starts(new)), cache.sta, 5000)
    cu = starts(new)
    for s in (0, 57, 199, 200, 201, 300):
        row = torch.tensor(cache.rows[s], device=DEV)
        for t, at in zip(cache.pool, (0, Hkv)):
            assert same(t[row].flatten(0, 1)[:new[s]].cpu(), x[cu[s]:cu[s + 1], at:at + Hkv])
