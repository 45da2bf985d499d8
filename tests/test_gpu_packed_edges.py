"""Attention over packed sequences at the edges of its arguments, against the definition in 64 bits; errors allowed as in test_gpu_packed."""
import math

import pytest
import torch

import paper_2502_04507_amd as sta
from tests import layer_util as lu
from tests.test_gpu_packed import BF, DEV, bounds, check, close, ints, randn, starts

pytestmark = pytest.mark.gpu

# Hq, Hkv, queries, keys, whether the launch is cut into parts: single tokens whole and in parts, two groups and four in a workgroup,
# tiles in parts, workgroups of four waves that share their stages
LSE = [(4, 2, [1, 3], [40, 70], False), (4, 2, [1, 2], [3000, 77], True), (16, 8, [300] * 4, [300] * 4, False), (6, 3, [70, 45, 300], [70, 45, 300], False),
       (8, 2, [100, 40], [4000, 300], True), (32, 16, [520] * 9, [520] * 9, False)]


def forward(q, k, v, lq, lk, parts=False, **kw):
    Hq, Hkv, D = q.shape[1], k.shape[1], q.shape[2]
    o, lse = torch.full_like(q, 7.0, device=DEV), torch.full((Hq, sum(lq)), 7.0, device=DEV)
    n = sta.sta_packed_workspace_bytes(Hq, Hkv, D, len(lq), sum(lq), max(lq), max(lk))
    assert (n > 0) or not parts
    sta.sta_packed_forward(q.to(DEV), k.to(DEV), v.to(DEV), o, ints(starts(lq)), ints(starts(lk)), max(lq), max(lk), lse=lse,
                           workspace=torch.empty(n, dtype=torch.uint8, device=DEV) if parts else None, **kw)
    return o, lse


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("which", ["q", "k"])
@pytest.mark.parametrize("case", LSE, ids=[str(i) for i in range(len(LSE))])
def test_lse_of_rows_that_meet_nan_is_nan(case, which, D):
    """-infinity is the mark of rows that see no key, and of no others; rows that meet no NaN keep their lse."""
    Hq, Hkv, lq, lk, parts = case
    g = Hq // Hkv
    q, k, v = randn((sum(lq), Hq, D), 1), randn((sum(lk), Hkv, D), 2), randn((sum(lk), Hkv, D), 3)
    for s in range(len(lq)):
        if which == "q":
            q[starts(lq)[s] + lq[s] - 1, g, 3] = float("nan")
        else:
            k[starts(lk)[s] + lk[s] - lq[s], 1, D - 1] = float("nan")            # the first row sees it
    o, lse = forward(q, k, v, lq, lk, parts)
    o, lse = o.cpu(), lse.cpu().double()
    for s in range(len(lq)):
        a, b = slice(starts(lq)[s], starts(lq)[s] + lq[s]), slice(starts(lk)[s], starts(lk)[s] + lk[s])
        Q, K, V = q[a].double(), k[b].double(), v[b].double()
        meets = torch.zeros((Hq, lq[s]), dtype=torch.bool)
        if which == "q":
            meets[g, -1] = True
        else:
            meets[g:2 * g] = True
        assert torch.equal(torch.isnan(lse[:, a]), meets), s
        assert torch.equal(torch.isnan(o[a]).all(-1).T, meets) and torch.equal(torch.isnan(o[a]).any(-1).T, meets), s
        _, want = lu.attention(Q.nan_to_num(0.0), K.nan_to_num(0.0), V, True, D ** -0.5)
        _, b_lse, _ = bounds(Q.nan_to_num(0.0), K.nan_to_num(0.0), V, True, D ** -0.5, want)
        assert bool(((lse[:, a] - want).abs() <= b_lse)[~meets].all()), s


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("which", ["q", "k"])
def test_gradients_of_rows_that_met_nan_in_the_forward(which, D):
    """NaN in q or k when o and lse are formed as well: the gradients of such rows and of all that they see are NaN, none is an infinity, other sequences
    and key heads keep their bits."""
    Hq, Hkv, lens = 6, 3, [70, 45, 300]
    T, cu = sum(lens), ints(starts(lens))
    at, head, kv = 70 + 20, 3, 1                            # token 20 of the second sequence
    x = [randn((T, h, D), i + 1) for i, h in enumerate((Hq, Hkv, Hkv))]
    d_o = randn((T, Hq, D), 4).to(DEV)
    results = []
    for bad in (False, True):
        if bad:
            x[which == "k"][at, kv if which == "k" else head, 5] = float("nan")
        o, lse = forward(*x, lens, lens)
        dev = [t.to(DEV) for t in x]
        d = [torch.empty_like(t) for t in dev]
        ws = torch.empty(sta.sta_packed_backward_workspace_bytes(Hq, T), dtype=torch.uint8, device=DEV)
        sta.sta_packed_backward(*dev, o, d_o, lse, *d, cu, cu, max(lens), max(lens), ws)
        results.append([t.cpu() for t in d])
    before, (dq, dk, dv) = results
    rows, keys = (slice(at, 115), slice(70, 115)) if which == "k" else (slice(at, at + 1), slice(70, at + 1))
    assert bool(torch.isnan(dq[rows, head]).all())
    assert bool(torch.isnan(dk[keys, kv]).all()) and bool(torch.isnan(dv[keys, kv]).all())
    assert not any(bool(torch.isinf(t).any()) for t in (dq, dk, dv))
    for a, b in zip((dq, dk, dv), before):
        a, b = (t.view(torch.int16).view(T, Hkv, -1, D) for t in (a, b))
        assert torch.equal(a[:70], b[:70]) and torch.equal(a[115:], b[115:])
        assert torch.equal(a[:, [0, 2]], b[:, [0, 2]])


# Hq, Hkv, queries, keys, max_q, max_k: few tiles and many, more sequences than a wave has lanes, keys' gradients cut along the rows, nothing at all
TOO_LOW = [(4, 2, [300, 20, 70], [300, 25, 70], 60, 300), (4, 2, [300, 20, 70], [200, 25, 90], 60, 50), (32, 16, [520] * 9 + [40], [520] * 9 + [40], 200, 520),
           (2, 2, [130, 1, 7] * 30, [130, 3, 5] * 30, 40, 130), (16, 1, [900, 600], [300, 5], 700, 300), (4, 2, [50, 3], [50, 9], 0, 50), (4, 2, [50, 3], [50, 9], 50, 0)]


@pytest.mark.parametrize("causal", [False, True])
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("case", TOO_LOW, ids=[str(i) for i in range(len(TOO_LOW))])
def test_gradients_where_bounds_of_lengths_are_too_low(case, D, causal):
    """Query tokens beyond max_q, and keys beyond max_k, may stay unwritten; what is written sums over the rows up to max_q, whatever the workspace held."""
    Hq, Hkv, lq, lk, max_q, max_k = case
    q, k, v, g = (randn((sum(n), h, D), i + 1) for i, (h, n) in enumerate(((Hq, lq), (Hkv, lk), (Hkv, lk), (Hq, lq))))
    x = [t.to(DEV) for t in (q, k, v)]
    o, lse = torch.empty_like(x[0]), torch.empty((Hq, sum(lq)), device=DEV)
    cu = ints(starts(lq)), ints(starts(lk))
    sta.sta_packed_forward(*x, o, *cu, max(lq), max(lk), causal=causal, lse=lse)
    results = []
    for held in (0, 255, 63):
        ws = torch.full((sta.sta_packed_backward_workspace_bytes(Hq, sum(lq)),), held, dtype=torch.uint8, device=DEV)
        d = [torch.full_like(t, 7.0) for t in x]
        sta.sta_packed_backward(*x, o, g.to(DEV), lse, *d, *cu, max_q, max_k, ws, causal=causal)
        results.append(d)
    for d in results[1:]:
        assert all(torch.equal(a.view(torch.int16), b.view(torch.int16)) for a, b in zip(d, results[0]))
    dq, dk, dv = (t.cpu() for t in results[0])
    c = D ** -0.5
    for s in range(len(lq)):
        a, b = slice(starts(lq)[s], starts(lq)[s] + lq[s]), slice(starts(lk)[s], starts(lk)[s] + lk[s])
        nq, nk = min(lq[s], max_q), min(lk[s], max_k)
        Q, K, V, G = q[a].double(), k[b].double(), v[b].double(), g[a].double()
        G[nq:] = 0.0                                        # rows that are left out add nothing
        _, want_lse, *want = lu.attention(Q, K, V, causal, c, G)
        _, _, off = bounds(Q, K, V, causal, c, want_lse, G)
        for name, got, w, e, n in (("dq", dq[a], want[0], off[0], nq), ("dk", dk[b], want[1], off[1], nk), ("dv", dv[b], want[2], off[2], nk)):
            close(got[:n], w[:n], e[:n], "sequence %d %s" % (s, name), norm=False)


@pytest.mark.parametrize("D", [64, 128])
def test_rows_within_bounds_that_are_too_low_are_written(D):
    """A sequence longer than max_q takes nothing from the others."""
    Hq, Hkv, lq, lk = 4, 2, [700, 60, 33, 60], [700, 60, 90, 61]
    q, k, v = randn((sum(lq), Hq, D), 1).to(DEV), randn((sum(lk), Hkv, D), 2).to(DEV), randn((sum(lk), Hkv, D), 3).to(DEV)
    o, right = torch.full_like(q, 7.0), torch.empty_like(q)
    sta.sta_packed_forward(q, k, v, o, ints(starts(lq)), ints(starts(lk)), 60, 90)
    sta.sta_packed_forward(q, k, v, right, ints(starts(lq)), ints(starts(lk)), 700, 700)
    for a, n in zip(starts(lq), lq):
        n = min(n, 60)
        assert float((o[a:a + n].float() - right[a:a + n].float()).abs().max()) < 2e-2


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("sign", [-1.0, 1.0])
@pytest.mark.parametrize("with_lse", [False, True])
@pytest.mark.parametrize("case", LSE, ids=[str(i) for i in range(len(LSE))])
def test_rows_whose_keys_all_have_the_lowest_or_largest_score(case, with_lse, sign, D):
    """Scores that a scale of 1 leaves finite, and whose products with log2(e) are not: all keys that a row sees count alike."""
    Hq, Hkv, lq, lk, parts = case
    g, most = Hq // Hkv, sign * torch.finfo(BF).max
    q, k, v = torch.zeros((sum(lq), Hq, D), dtype=BF), randn((sum(lk), Hkv, D), 2), randn((sum(lk), Hkv, D), 3)
    q[..., 0], k[..., 0] = 1.0, most
    o, lse = torch.full_like(q, 7.0, device=DEV), torch.full((Hq, sum(lq)), 7.0, device=DEV) if with_lse else None
    n = sta.sta_packed_workspace_bytes(Hq, Hkv, D, len(lq), sum(lq), max(lq), max(lk))
    sta.sta_packed_forward(q.to(DEV), k.to(DEV), v.to(DEV), o, ints(starts(lq)), ints(starts(lk)), max(lq), max(lk), scale=1.0, lse=lse,
                           workspace=torch.empty(n, dtype=torch.uint8, device=DEV) if parts else None)
    for s in range(len(lq)):
        a, b = starts(lq)[s], starts(lk)[s]
        seen = lk[s] - lq[s] + 1 + torch.arange(lq[s])
        V = v[b:b + lk[s]].double()
        want = (V.cumsum(0)[seen - 1] / seen[:, None, None]).repeat_interleave(g, 1)
        size = (V.abs().cumsum(0)[seen - 1] / seen[:, None, None]).repeat_interleave(g, 1)
        close(o[a:a + lq[s]], want, (2.0 ** -7 + 2.0 ** -11) * size, "sequence %d" % s, norm=False)
    if with_lse:
        assert bool((lse == most).all())                    # ln of how many is far below the spacing there


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("with_lse", [False, True])
@pytest.mark.parametrize("case", LSE, ids=[str(i) for i in range(len(LSE))])
def test_a_scale_next_to_nothing(case, with_lse, D):
    """Every key that a row sees counts alike."""
    Hq, Hkv, lq, lk, parts = case
    q, k, v = randn((sum(lq), Hq, D), 1), randn((sum(lk), Hkv, D), 2), randn((sum(lk), Hkv, D), 3)
    o, lse = torch.full_like(q, 7.0, device=DEV), torch.full((Hq, sum(lq)), 7.0, device=DEV) if with_lse else None
    n = sta.sta_packed_workspace_bytes(Hq, Hkv, D, len(lq), sum(lq), max(lq), max(lk))
    sta.sta_packed_forward(q.to(DEV), k.to(DEV), v.to(DEV), o, ints(starts(lq)), ints(starts(lk)), max(lq), max(lk), scale=1e-38, lse=lse,
                           workspace=torch.empty(n, dtype=torch.uint8, device=DEV) if parts else None)
    for s in range(len(lq)):
        a, b = starts(lq)[s], starts(lk)[s]
        seen = lk[s] - lq[s] + 1 + torch.arange(lq[s])
        V = v[b:b + lk[s]].double()
        want = (V.cumsum(0)[seen - 1] / seen[:, None, None]).repeat_interleave(Hq // Hkv, 1)
        size = (V.abs().cumsum(0)[seen - 1] / seen[:, None, None]).repeat_interleave(Hq // Hkv, 1)
        close(o[a:a + lq[s]], want, (2.0 ** -7 + 2.0 ** -11) * size, "sequence %d" % s, norm=False)
        if with_lse:
            off = (lse[:, a:a + lq[s]].cpu().double() - torch.log(seen.double())).abs()
            assert bool((off <= 2.0 ** -20 * (1 + torch.log(seen.double())) + lk[s] * 2.0 ** -24).all())


@pytest.mark.parametrize("causal", [False, True])
@pytest.mark.parametrize("D", [64, 128])
def test_hundreds_of_sequences_of_uneven_lengths(D, causal):
    """More sequences than four waves have lanes, some without rows or keys, a few long: forward and gradients."""
    lq = [(7 * i * i) % 41 if i % 97 else 300 for i in range(330)]
    lk = [(5 * i * i + 3) % 47 if i % 61 else 257 for i in range(330)]
    assert 0 in lq and 0 in lk and max(lq) == 300
    check(2, 1, D, lq, lk, causal, train=True)
    check(2, 1, D, lq, lk, causal)


@pytest.mark.parametrize("Hq,Hkv,n,m,causal", [(4, 2, 200, 200, True), (16, 1, 900, 70, False)])
def test_a_training_step_in_a_graph(Hq, Hkv, n, m, causal):
    """Forward and gradients, the keys' cut along the rows in the second, with inputs and lengths that change between replays."""
    D = 64
    x = [torch.empty((t, h, D), dtype=BF, device=DEV) for t, h in ((n, Hq), (m, Hkv), (m, Hkv), (n, Hq))]
    cu_q, cu_k = ints([0, n // 2, n]), ints([0, m // 2, m])
    outs = [[torch.zeros_like(t) for t in (x[0], *x[:3])] + [torch.zeros((Hq, n), device=DEV)] for _ in range(2)]
    ws = [torch.empty(sta.sta_packed_backward_workspace_bytes(Hq, n), dtype=torch.uint8, device=DEV) for _ in range(2)]

    def step(i):
        o, dq, dk, dv, lse = outs[i]
        sta.sta_packed_forward(*x[:3], o, cu_q, cu_k, n, m, causal=causal, lse=lse)
        sta.sta_packed_backward(*x[:3], o, x[3], lse, dq, dk, dv, cu_q, cu_k, n, m, ws[i], causal=causal)

    for t in x:
        t.zero_()
    step(0)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step(0)
    for seed, at in enumerate((n // 2, 3, n - 1)):
        for i, t in enumerate(x):
            t.copy_(randn(t.shape, 10 * seed + i))
        cu_q.copy_(torch.tensor([0, at, n], dtype=torch.int32))
        cu_k.copy_(torch.tensor([0, min(at, m - 1), m], dtype=torch.int32))
        ws[0].fill_(255)
        graph.replay()
        torch.cuda.synchronize()
        step(1)
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(*outs)), at
