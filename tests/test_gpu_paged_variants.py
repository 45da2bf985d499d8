"""Kernels of the operators on a cache in pages that launches of many sequences or of large ones take, and scales that the caller gives, on the GPU, against plain implementations in 64
bits with the errors that test_gpu_packed and test_gpu_paged_weights derive."""
import pytest
import torch

import paper_2502_04507_amd as sta
from tests import layer_util as lu
from tests.paged_util import DEV, Cache, forward, ints, same, starts
from tests.test_gpu_packed import bounds, close, randn
from tests.test_gpu_paged_weights import check_weights

pytestmark = pytest.mark.gpu

MANY = [33 + 7 * i % 20 for i in range(70)]             # new tokens of 70 sequences
KEYS = [n + 37 * i % 261 for i, n in enumerate(MANY)]

# Hq, Hkv, D, new, used, causal, page, decay.  Workgroups for a sequence and key head: one for 256 keys where those make two a CU, else for 128 or 64
WEIGHTS = {
    "two of 64 channels, 256 keys a workgroup": (16, 16, 64, [64, 40], [5000, 4200], True, 16, 0.5),
    "two of 64 channels, 256 keys a workgroup, not causal": (16, 16, 64, [33, 500], [4700, 4099], False, 7, 0.0),
    "70 of 128 channels, 256 keys": (4, 4, 128, MANY, KEYS, True, 3, 1.0),
    "70 of 128 channels, 256 keys, groups of two": (8, 4, 128, MANY, KEYS, False, 16, 0.5),
    "70 of 64 channels, 256 keys": (4, 4, 64, MANY, KEYS, True, 5, 0.75),
    "70 of 64 channels, 256 keys, groups of three": (12, 4, 64, MANY, KEYS, True, 24, 1.0),
    "70 of 128 channels, 128 keys": (2, 1, 128, MANY, KEYS, True, 16, 1.0),
    "70 of 64 channels, 128 keys": (3, 1, 64, MANY, KEYS, True, 9, 0.5),
    "70 of 64 channels, more than 512 rows": (4, 4, 64, [513] + MANY[1:], [600] + KEYS[1:], True, 16, 1.0),
    "66 of 128 channels, 64 keys": (1, 1, 128, [40] * 66, [41 + i for i in range(66)], True, 8, 1.0),
    "66 of 64 channels, 64 keys": (2, 1, 64, [40] * 66, [41 + i for i in range(66)], True, 1, 1.0),
    "100 of few rows": (8, 2, 64, [1, 2, 0, 4] * 25, [1 + 91 * i % 700 for i in range(100)], True, 16, 0.5),
    "100 of few rows of 128 channels": (8, 2, 128, [1, 8, 0, 4] * 25, [8 + 91 * i % 700 for i in range(100)], True, 16, 0.5),
}


@pytest.mark.parametrize("name", WEIGHTS)
def test_weights(name):
    Hq, Hkv, D, new, used, causal, page, decay = WEIGHTS[name]
    cache = Cache(Hkv, D, page, used, seed=31)
    q = randn((sum(new), Hq, D), 33)
    _, lse = forward(q.to(DEV), cache, new, causal=causal, lse=True)
    check_weights(cache, q, lse, new, causal, decay)


# single tokens whole and in parts; tiles by two groups, by four, in parts, and shared by four waves
SHAPES = [(4, 2, [1, 3], [40, 70]), (4, 2, [1, 2], [3000, 77]), (16, 8, [300] * 4, [300] * 4), (6, 3, [70, 45, 300], [70, 45, 300]), (8, 2, [100, 40], [9000, 300]), (32, 16, [520] * 9, [520] * 9)]


@pytest.mark.parametrize("scale", [0.37, 0.004])
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("shape", SHAPES, ids=[str(i) for i in range(len(SHAPES))])
def test_a_scale_of_the_callers(shape, D, scale):
    """Not 1 / sqrt(D), which 0 stands for; by the extension and the general path."""
    Hq, Hkv, new, used = shape
    cache = Cache(Hkv, D, 16, used, seed=35)
    q = randn((sum(new), Hq, D), 37)
    c = float(torch.tensor(scale, dtype=torch.float32))         # as the library takes it
    o, lse = forward(q.to(DEV), cache, new, scale=scale, lse=True)
    cu = starts(new)
    for s in range(len(new)):
        a = slice(cu[s], cu[s + 1])
        Q, K, V = q[a].double(), cache.k[s].double(), cache.v[s].double()
        want = lu.attention(Q, K, V, True, c)
        b_o, b_lse, _ = bounds(Q, K, V, True, c, want[1])
        close(o[a], want[0], b_o, "sequence %d" % s)
        assert bool(((lse[:, a].cpu().double() - want[1]).abs() <= b_lse).all()), s
    w = check_weights(cache, q, lse, new, scale=scale, before=False)
    stream = torch.cuda.current_stream()
    args = (ints(cu), cache.sta, max(new), max(used))
    o2, w2 = torch.empty_like(o), torch.full_like(w, 7.0)
    n = sta.sta_paged_workspace_bytes(Hq, Hkv, D, len(new), sum(new), max(new), max(used))
    sta.sta_paged_forward(q.to(DEV), o2, *args, scale=scale, lse=lse.clone(), workspace=torch.empty(max(n, 16), dtype=torch.uint8, device=DEV), stream=stream)
    sta.sta_paged_weights(q.to(DEV), lse, w2, *args, scale=scale, stream=stream)
    assert same(o, o2) and same(w, w2)


def test_a_step_beyond_the_table():
    """Six tokens, two of which the table has no place for: the rows of the first four are keys, and the attention and the weights take the six for the last of the keys there are."""
    Hq, Hkv, D, page, room = 4, 2, 64, 16, 48
    cache = Cache(Hkv, D, page, [room], seed=41, room=3)
    x, q = randn((6, 2 * Hkv, D), 42).to(DEV), randn((6, Hq, D), 43).to(DEV)
    cache.lengths.fill_(room + 2)
    sta.sta_paged_append(x[:, :Hkv], x[:, Hkv:], ints([0, 6]), cache.sta, 6)
    for t, new in ((cache.k[0], x[:, :Hkv]), (cache.v[0], x[:, Hkv:])):
        t[room - 4:] = new[:4].cpu()
    at = [cache.place(0, j) for j in range(room)]
    for t, rows in zip(cache.pool, (cache.k[0], cache.v[0])):
        assert same(torch.stack([t[p, s] for p, s in at]).cpu(), rows)
    beyond, within = [], []
    for out in (beyond, within):
        o, lse = forward(q, cache, [6], lse=True, max_k=room + 2)
        w = torch.zeros((cache.pages, Hkv, page), device=DEV)
        sta.sta_paged_weights(q, lse, w, ints([0, 6]), cache.sta, 6, room + 2)
        out += [o, lse, w]
        cache.lengths.fill_(room)
    assert all(same(a, b) for a, b in zip(beyond, within))
    want = lu.attention(q.cpu().double(), cache.k[0].double(), cache.v[0].double(), True, D ** -0.5)
    b_o, _, _ = bounds(q.cpu().double(), cache.k[0].double(), cache.v[0].double(), True, D ** -0.5, want[1])
    close(beyond[0], want[0], b_o, "beyond")
