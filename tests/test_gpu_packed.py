"""Attention over packed sequences on the GPU, against the definition in 64 bits.

Allowed errors, worst cases of each step (inputs are the same bf16 numbers on both sides):
  scores     products of bf16 numbers are exact in fp32, the sum of D of them is off by (D + 4) 2^-24 of the sum of the absolute
             products; e_s is that times the scale, at most 2e-3 on these inputs, and a relative error of the probability;
  O          probabilities are rounded to bf16 (2^-8) and, where no lse is asked for, so is their sum: (2^-7 + 2 e_s + 2^-11) sum_j P_ij |V_j|,
             and one rounding of the result;
  lse        e_s, the sum of lk terms (lk 2^-24), a logarithm and a product (2^-21 + 2^-21 |lse|);
  dV         (2^-8 + e_s + 2^-11) sum_i P_ij |dO_i|;
  dS         P_ij times what delta_i is off by, dO_i . (error of O_i), and of |P_ij| (|dP_ij| + |delta_i|) the relative errors of P (e_s + 2^-11) and
             one rounding of dS to bf16 (2^-8); dQ and dK: that times |K| and |Q|, summed.
The relative 2-norm of the error stays below 1e-2 besides, where rows see enough keys for the result not to cancel."""
import math

import pytest
import torch

import paper_2502_04507_amd as sta
from tests import layer_util as lu

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
BF = torch.bfloat16


def randn(shape, seed, spread=1.0):
    return (torch.randn(shape, generator=torch.Generator().manual_seed(seed)) * spread).to(BF)


def starts(lengths):
    out = [0]
    for n in lengths:
        out.append(out[-1] + n)
    return out


def ints(x):
    return torch.tensor(x, dtype=torch.int32, device=DEV)


def bounds(q, k, v, causal, scale, lse, d_o=None):
    """Of one sequence: what O, lse (and the gradients) may be off by."""
    lq, Hq, D = q.shape
    lk, Hkv = k.shape[0], k.shape[1]
    keep = lu.seen(lq, lk, causal)
    b_o, b_lse = torch.zeros_like(q), torch.zeros((Hq, lq), dtype=torch.float64)
    b = [torch.zeros_like(x) for x in (q, k, v)]
    for h in range(Hq):
        n = h // (Hq // Hkv)
        if lq == 0 or lk == 0:
            continue
        Q, K, V = q[:, h], k[:, n], v[:, n]
        s = torch.where(keep, Q @ K.T * scale, -math.inf)
        p = torch.where(keep, torch.exp(s - torch.where(torch.isinf(lse[h]), 0.0, lse[h])[:, None]), 0.0)
        e_s = torch.where(keep, (D + 4) * 2.0 ** -24 * (Q.abs() @ K.abs().T) * scale, 0.0).amax(-1, keepdim=True)
        assert float(e_s.max()) < 2e-3
        b_lse[h] = e_s[:, 0] + lk * 2.0 ** -24 + 2.0 ** -21 + 2.0 ** -21 * torch.where(torch.isinf(lse[h]), 0.0, lse[h]).abs()
        off = (2.0 ** -7 + 2 * e_s + 2.0 ** -11) * (p @ V.abs())
        b_o[:, h] = off
        if d_o is None:
            continue
        G, o = d_o[:, h], p @ V
        b[2][:, n] += (p * (2.0 ** -8 + e_s + 2.0 ** -11)).T @ G.abs()
        dP, delta = G @ V.T, (G * o).sum(-1, keepdim=True)
        e_delta = (G.abs() * (off + 2.0 ** -8 * (o.abs() + off))).sum(-1, keepdim=True)
        e_ds = p * e_delta + p * (dP.abs() + delta.abs()) * (2.0 ** -8 + e_s + 2.0 ** -11)
        b[0][:, h] = e_ds @ K.abs() * scale
        b[1][:, n] += e_ds.T @ Q.abs() * scale
    return b_o, b_lse, b


def close(got, want, slack, label, norm=True):
    lu.assert_rounded(got, want, slack + 1e-30, label)
    if norm and want.numel() and float(want.norm()) > 0:
        rel = float((got.cpu().double() - want).norm() / want.norm())
        assert rel < 1e-2, "%s: relative 2-norm %.2e" % (label, rel)


def check(Hq, Hkv, D, lq, lk, causal, train=False, scale=0.0, workspace=True, cache=0, spread=1.0, layout="packed", seed=1):
    tq, slots = sum(lq), [cache] * len(lk) if cache else lk
    tk = sum(slots)
    q, k, v, g = randn((tq, Hq, D), seed, spread), randn((tk, Hkv, D), seed + 1, spread), randn((tk, Hkv, D), seed + 2), randn((tq, Hq, D), seed + 3)
    cu_q, cu_k = starts(lq), starts(slots)

    def dev(x):
        if layout == "heads":               # [heads, tokens, D]
            return x.transpose(0, 1).contiguous().to(DEV).transpose(0, 1)
        if layout == "wide":                # rows of a wider tensor
            y = torch.full((x.shape[0], x.shape[1] + 2, D + 8), float("nan"), dtype=BF)
            y[:, 1:-1, 8:] = x
            return y.to(DEV)[:, 1:-1, 8:]
        return x.to(DEV)

    qd, kd, vd, gd = (dev(x) for x in (q, k, v, g))
    if cache:                               # what is not used of a slot is nobody's
        for s, n in enumerate(lk):
            kd[cu_k[s] + n:cu_k[s + 1]] = float("nan")
            vd[cu_k[s] + n:cu_k[s + 1]] = float("inf")
    o = dev(torch.full_like(q, float("nan")))
    lse = torch.full((Hq, tq), float("nan"), device=DEV) if train else None
    ws = None
    max_q, max_k = max(lq), max(lk)
    if workspace:
        n = sta.sta_packed_workspace_bytes(Hq, Hkv, D, len(lq), tq, max_q, max_k)
        ws = torch.full((max(n, 16),), 255, dtype=torch.uint8, device=DEV)
    args = (ints(cu_q), ints(cu_k), max_q, max_k)
    for once in range(2):
        sta.sta_packed_forward(qd, kd, vd, o, *args, causal=causal, scale=scale, lse=lse, k_used=ints(lk) if cache else None, workspace=ws)
        now = o.clone()
        assert once == 0 or torch.equal(now.view(torch.int16), before.view(torch.int16))
        before = now
    if train:
        dq, dk, dv = (dev(torch.full_like(x, float("nan"))) for x in (q, k, v))
        ws = torch.full((sta.sta_packed_backward_workspace_bytes(Hq, tq),), 255, dtype=torch.uint8, device=DEV)
        before = None
        for once in range(2):
            sta.sta_packed_backward(qd, kd, vd, o, gd, lse, dq, dk, dv, *args, ws, causal=causal, scale=scale)
            now = [x.clone() for x in (dq, dk, dv)]
            assert before is None or all(torch.equal(a, b) for a, b in zip(before, now))
            before = now
    c = scale if scale > 0 else D ** -0.5
    for s in range(len(lq)):
        a, b = slice(cu_q[s], cu_q[s] + lq[s]), slice(cu_k[s], cu_k[s] + lk[s])
        Q, K, V, G = q[a].double(), k[b].double(), v[b].double(), g[a].double()
        want = lu.attention(Q, K, V, causal, c, G if train else None)
        b_o, b_lse, b_d = bounds(Q, K, V, causal, c, want[1], G if train else None)
        label = "sequence %d (%d, %d)" % (s, lq[s], lk[s])
        close(o[a], want[0], b_o, label + " o")
        if not train:
            continue
        got = lse[:, a].cpu().double()
        assert torch.equal(torch.isinf(got), torch.isinf(want[1])) and not bool(torch.isnan(got).any()), label
        seen = ~torch.isinf(want[1])
        assert bool(((got - want[1]).abs()[seen] <= b_lse[seen]).all()), label
        for name, x, i, r in (("dq", dq, 2, a), ("dk", dk, 3, b), ("dv", dv, 4, b)):
            close(x[r], want[i], b_d[i - 2], label + " " + name, norm=lk[s] >= 32 and lq[s] >= 32)


CASES = [
    # Hq, Hkv, D, queries, keys, causal
    (1, 1, 64, [1], [1], True), (2, 1, 128, [1, 1], [1, 5], True), (4, 4, 64, [5], [5], False), (4, 2, 128, [31, 32, 33], [31, 32, 33], True),
    (3, 1, 64, [64, 65, 63], [64, 65, 63], True), (5, 5, 128, [127, 1, 128, 129], [127, 1, 128, 129], True), (8, 8, 64, [200, 7], [200, 7], False),
    (6, 2, 128, [40, 0, 17], [40, 9, 0], True), (6, 2, 128, [40, 0, 17], [40, 9, 0], False), (5, 1, 64, [90], [33], True), (10, 2, 128, [100, 3], [37, 1], True),
    (4, 1, 128, [33, 100], [300, 101], True), (16, 1, 64, [3, 130], [70, 130], True), (8, 1, 128, [70], [257], False), (1, 1, 128, [300], [300], True),
    (12, 12, 64, [77, 12, 1], [77, 12, 1], False), (7, 1, 64, [19, 37], [50, 37], True), (2, 2, 64, [1] * 70 + [40], [1] * 70 + [45], True),
    (3, 3, 128, [2] * 130, [3] * 130, True), (9, 3, 64, [513], [513], True), (40, 8, 128, [9, 60], [9, 61], True),
]


@pytest.mark.parametrize("train", [False, True])
@pytest.mark.parametrize("case", CASES, ids=[str(i) for i in range(len(CASES))])
def test_against_64_bits(case, train):
    check(*case, train=train)


# few rows a sequence: the bounds of 16 and 32 rows, lengths around a sub-block and around four waves' shares, parts with and without room
FEW = [
    (4, 1, 128, [1, 1, 1], [1, 31, 1700], 1700), (8, 8, 64, [1] * 5, [5, 64, 129, 2100, 1], 2176), (16, 1, 64, [1, 1], [2000, 33], 2000), (32, 2, 128, [1], [700], 704),
    (8, 1, 128, [2, 4], [130, 1500], 1600), (8, 1, 64, [3, 1], [3, 2500], 2501), (5, 1, 128, [4, 6, 1], [4, 600, 90], 640), (2, 2, 64, [9, 32], [1100, 33], 1200),
    (24, 24, 128, [1, 2], [520, 4000], 4000), (33, 1, 64, [1], [1033], 1033), (4, 2, 128, [1, 0, 1], [0, 40, 9], 64),
]


@pytest.mark.parametrize("workspace", [False, True])
@pytest.mark.parametrize("case", FEW, ids=[str(i) for i in range(len(FEW))])
def test_few_rows_against_a_cache(case, workspace):
    Hq, Hkv, D, lq, lk, cache = case
    check(Hq, Hkv, D, lq, lk, True, workspace=workspace, cache=cache)


@pytest.mark.parametrize("D", [64, 128])
def test_few_rows_with_lse_and_parts(D):
    Hq, Hkv, lq, lk = 8, 2, [1, 3], [3000, 77]
    check(Hq, Hkv, D, lq, lk, True, train=True)


@pytest.mark.parametrize("case", [
    (4, 1, 128, [100, 260], [3000, 2049], 3008), (3, 3, 64, [200], [1800], 1800), (8, 2, 128, [40], [5000], 5000), (2, 1, 64, [129, 17, 300], [4097, 17, 301], 4100),
    (8, 2, 128, [70, 150], [9000, 100], 9000), (2, 2, 64, [300], [8200], 8200), (2, 2, 64, [1, 70, 0], [8300, 8191, 300], 8300),
])
def test_tiles_cut_along_the_keys(case):
    Hq, Hkv, D, lq, lk, cache = case
    assert sta.sta_packed_workspace_bytes(Hq, Hkv, D, len(lq), sum(lq), max(lq), max(lk)) > 0
    check(Hq, Hkv, D, lq, lk, True, cache=cache)
    check(Hq, Hkv, D, lq, lk, False, cache=cache)


# Launches that fill the chip: workgroups of four waves of rows, or of keys, in one walk; more sequences than a wave has lanes.
@pytest.mark.parametrize("case", [
    (12, 12, 64, [260] * 30 + [1, 0, 129] + [256] * 37, None, True), (16, 8, 128, [258] * 64, None, True), (8, 8, 128, [300, 290] * 32, [270, 310] * 32, False),
])
def test_large_launches(case):
    Hq, Hkv, D, lq, lk, causal = case
    check(Hq, Hkv, D, lq, lk or lq, causal, train=True)
    check(Hq, Hkv, D, lq, lk or lq, causal)


# Between a few tiles and a full chip: one wave, or two, of rows (keys) by four, or two, groups.
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("case", [(4, 2, [300], [300], True), (6, 2, [290, 1, 40], [257, 300, 0], False), (16, 16, [300] * 4, [300] * 4, True), (20, 10, [513, 33, 700], [500, 270, 733], True)])
def test_walk_groups(case, D):
    Hq, Hkv, lq, lk, causal = case
    check(Hq, Hkv, D, lq, lk, causal, train=True)
    check(Hq, Hkv, D, lq, lk, causal)


# Few keys that many rows see: their gradients in parts of the rows.
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("causal", [False, True])
@pytest.mark.parametrize("case", [(16, 1, [600, 3, 0], [300, 5, 9]), (24, 2, [700], [129]), (16, 1, [0, 530, 515], [70, 77, 400]), (8, 1, [1300], [1300]), (1, 1, [9000], [40])])
def test_gradients_of_keys_cut_along_the_rows(case, causal, D):
    Hq, Hkv, lq, lk = case
    assert sta.sta_packed_backward_workspace_bytes(Hq, sum(lq)) > 2 * 4 * (Hq * sum(lq) + 64) + 16
    check(Hq, Hkv, D, lq, lk, causal, train=True)


@pytest.mark.parametrize("layout", ["heads", "wide"])
@pytest.mark.parametrize("D", [64, 128])
def test_layouts(layout, D):
    check(6, 3, D, [70, 1, 33], [90, 1, 33], True, train=True, layout=layout)
    check(4, 2, D, [1, 2], [90, 700], True, layout=layout)


@pytest.mark.parametrize("scale", [0.02, 0.7])
def test_scale(scale):
    check(4, 2, 64, [150], [150], True, train=True, scale=scale)


def test_large_scores_that_keep_growing():
    """Keys whose scores rise along the sequence by far more than the rescaling threshold, and fall again."""
    D, n = 64, 300
    q, v = torch.ones((n, 1, D), dtype=BF), randn((n, 1, D), 5)
    ramp = torch.cat([torch.linspace(-40, 60, 200), torch.linspace(60, -90, 100)])
    k = (ramp[:, None, None] / 8.0).expand(n, 1, D).to(BF).contiguous()
    o = torch.empty_like(q, device=DEV)
    sta.sta_packed_forward(q.to(DEV), k.to(DEV), v.to(DEV), o, ints([0, n]), ints([0, n]), n, n, causal=True)
    want, lse = lu.attention(q.double(), k.double(), v.double(), True, 0.125)
    p_v = torch.zeros_like(want)
    s = torch.where(lu.seen(n, n, True), q[:, 0].double() @ k[:, 0].double().T * 0.125, -math.inf)
    p_v[:, 0] = torch.exp(s - lse[0][:, None]) @ v[:, 0].double().abs()
    close(o, want, (2.0 ** -7 + 4e-3 + 2.0 ** -11) * p_v, "growing", norm=False)


def test_keys_of_the_lowest_number_first():
    """Keys masked through a channel: scores of the lowest numbers before ordinary ones."""
    D, n = 64, 150
    q, k, v = randn((n, 2, D), 1), randn((n, 1, D), 2), randn((n, 1, D), 3)
    q[..., 0] = 1.0
    k[:100, :, 0] = torch.finfo(BF).min
    k[100:, :, 0] = 0.0
    o = torch.empty_like(q, device=DEV)
    sta.sta_packed_forward(q.to(DEV), k.to(DEV), v.to(DEV), o, ints([0, n]), ints([0, n]), n, n, causal=False)
    want, lse = lu.attention(q.double(), k[100:].double(), v[100:].double(), False, 0.125)
    b_o, _, _ = bounds(q.double(), k[100:].double(), v[100:].double(), False, 0.125, lse)
    close(o, want, b_o, "lowest")


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("few", [False, True])
def test_no_number_of_an_unseen_key_reaches_a_row(D, few):
    """Values (and keys) of tokens that a row does not see hold infinities and NaN: in its own sequence later on, and in the neighbours."""
    Hq, Hkv = (4, 2) if few else (6, 3)
    lq, lk = ([5, 3], [40, 70]) if few else ([100, 70], [100, 90])
    q, k, v = randn((sum(lq), Hq, D), 1), randn((sum(lk), Hkv, D), 2), randn((sum(lk), Hkv, D), 3)
    bad = {}
    for s, (a, n) in enumerate(zip(starts(lk), lk)):
        for back, value in ((1, float("nan")), (2, float("inf")), (3, -float("inf"))):
            at = n - back
            bad[(s, at)] = value
            v[a + at, :, ::back] = value
            if back == 1:
                k[a + at, :, 1] = value
    o = torch.full(q.shape, 7.0, dtype=BF, device=DEV)
    n = sta.sta_packed_workspace_bytes(Hq, Hkv, D, 2, sum(lq), max(lq), max(lk))
    sta.sta_packed_forward(q.to(DEV), k.to(DEV), v.to(DEV), o, ints(starts(lq)), ints(starts(lk)), max(lq), max(lk), causal=True,
                           workspace=torch.empty(max(n, 16), dtype=torch.uint8, device=DEV))
    o = o.cpu()
    for s in range(2):
        a, b = starts(lq)[s], starts(lk)[s]
        for i in range(lq[s]):
            seen = i + 1 + lk[s] - lq[s]
            Q, K, V = q[a + i:a + i + 1].double(), k[b:b + seen].double(), v[b:b + seen].double()
            if seen == lk[s]:
                assert not bool(torch.isfinite(o[a + i]).all())
                continue
            K = K.nan_to_num(0.0)
            finite = torch.isfinite(V)
            want, lse = lu.attention(Q, K, torch.where(finite, V, 0.0), False, D ** -0.5)
            b_o, _, _ = bounds(Q, K, torch.where(finite, V, 0.0), False, D ** -0.5, lse)
            want_kind = torch.where(finite, 0.0, V).sum(0)                      # [Hkv, D]: 0, an infinity
            want_kind = want_kind.repeat_interleave(Hq // Hkv, 0)
            number = want_kind == 0
            got = o[a + i]
            assert torch.equal(torch.isnan(got), torch.isnan(want_kind)), (s, i)        # both infinities in one channel
            infinite = torch.isinf(want_kind)
            assert torch.equal(got.double()[infinite], want_kind[infinite]), (s, i)
            x = torch.where(number, got, torch.zeros_like(got))[None]
            lu.assert_rounded(x, torch.where(number, want[0], 0.0)[None], b_o + 1e-30, "row %d of %d" % (i, s))


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("which", [0, 1, 2, 3])
def test_no_number_leaves_its_sequence_and_head_in_the_gradients(which, D):
    """One value of q, k, v or d_o of the middle sequence is no number: the gradients of other sequences and key heads keep their bits."""
    Hq, Hkv, lens = 6, 3, [70, 45, 300]
    T, cu, kv = sum(lens), ints(starts(lens)), 1
    clean = [randn((T, h, D), i + 1).to(DEV) for i, h in enumerate((Hq, Hkv, Hkv, Hq))]
    o, lse = torch.empty_like(clean[0]), torch.empty((Hq, T), device=DEV)
    sta.sta_packed_forward(*clean[:3], o, cu, cu, max(lens), max(lens), lse=lse)
    ws = torch.empty(sta.sta_packed_backward_workspace_bytes(Hq, T), dtype=torch.uint8, device=DEV)
    results = []
    for value in (None, float("nan"), float("inf")):
        x = [t.clone() for t in clean]
        if value is not None:
            x[which][70 + 44, kv * (1 if which in (1, 2) else 2), 5] = value
        d = [torch.empty_like(t) for t in x[:3]]
        sta.sta_packed_backward(*x[:3], o, x[3], lse, *d, cu, cu, max(lens), max(lens), ws)
        results.append(d)
    for d in results[1:]:
        for a, b in zip(d, results[0]):
            g = a.shape[1] // Hkv
            a, b = (t.cpu().view(torch.int16).view(T, Hkv, g, D) for t in (a, b))
            assert torch.equal(a[:70], b[:70]) and torch.equal(a[115:], b[115:])
            assert torch.equal(a[:, [0, 2]], b[:, [0, 2]])


def test_rows_outside_every_sequence_are_left_alone():
    q, k, v = randn((50, 2, 64), 1).to(DEV), randn((60, 2, 64), 2).to(DEV), randn((60, 2, 64), 3).to(DEV)
    o = torch.full_like(q, 3.0)
    sta.sta_packed_forward(q, k, v, o, ints([5, 20, 40]), ints([0, 30, 50]), 20, 30)
    assert bool((o[:5] == 3).all()) and bool((o[40:] == 3).all()) and not bool((o[5:40] == 3).all(-1).any())


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("n", [3, 200])
def test_no_keys_and_no_queries_at_all(n, D):
    """Tensors without a token: rows that see nothing are 0 with lse -infinity, gradients of keys that nothing saw are 0."""
    x, none, two = randn((n, 4, D), 1).to(DEV), torch.empty((0, 2, D), dtype=BF, device=DEV), ints([0, n, n])
    o, lse, dq = torch.full_like(x, 3.0), torch.zeros((4, n), device=DEV), torch.full_like(x, 3.0)
    sta.sta_packed_forward(x, none, none, o, two, ints([0, 0, 0]), n, 0, lse=lse)
    assert bool((o == 0).all()) and bool((lse == -float("inf")).all())
    ws = torch.empty(sta.sta_packed_backward_workspace_bytes(4, n), dtype=torch.uint8, device=DEV)
    sta.sta_packed_backward(x, none, none, o, x, lse, dq, none.clone(), none.clone(), two, ints([0, 0, 0]), n, 0, ws)
    assert bool((dq == 0).all())
    q0, k = torch.empty((0, 4, D), dtype=BF, device=DEV), randn((n, 2, D), 2).to(DEV)
    dk, dv = torch.full_like(k, 3.0), torch.full_like(k, 3.0)
    sta.sta_packed_forward(q0, k, k, q0.clone(), ints([0, 0, 0]), two, 0, n)
    sta.sta_packed_backward(q0, k, k, q0, q0, torch.empty((4, 0), device=DEV), q0.clone(), dk, dv, ints([0, 0, 0]), two, 0, n, ws)
    assert bool((dk == 0).all()) and bool((dv == 0).all())


def test_bounds_that_leave_the_tensors_are_cut():
    """Wrong bounds: no access leaves the tensors, and sequences that are right keep their results."""
    q, k, v = randn((40, 2, 64), 1).to(DEV), randn((40, 2, 64), 2).to(DEV), randn((40, 2, 64), 3).to(DEV)
    good, o = torch.empty_like(q), torch.empty_like(q)
    sta.sta_packed_forward(q, k, v, good, ints([0, 20, 40]), ints([0, 20, 40]), 20, 20)
    sta.sta_packed_forward(q, k, v, o, ints([0, 20, 1000000]), ints([0, 20, 2000000]), 20, 20)
    assert torch.equal(o, good)
    sta.sta_packed_forward(q, k, v, o, ints([0, 20, -5]), ints([0, 20, -7]), 20, 20)
    assert torch.equal(o[:20], good[:20])


@pytest.mark.parametrize("D", [64, 128])
def test_lengths_beyond_max_q_leave_the_workspace(D):
    """Bounds that are too low: rows may stay unwritten, nothing outside the workspace is written, and what is written is right."""
    Hq, Hkv, lq, lk, most = 8, 2, [300, 290, 310], [9000, 8000, 8500], 60
    q, k, v = randn((sum(lq), Hq, D), 1).to(DEV), randn((sum(lk), Hkv, D), 2).to(DEV), randn((sum(lk), Hkv, D), 3).to(DEV)
    n = sta.sta_packed_workspace_bytes(Hq, Hkv, D, 3, sum(lq), most, max(lk))
    assert n > 0
    room = torch.full((n + (256 << 20),), 77, dtype=torch.uint8, device=DEV)
    args = (q, k, v), (ints(starts(lq)), ints(starts(lk)))
    o, right = (torch.full_like(q, float("nan")) for _ in range(2))
    sta.sta_packed_forward(*args[0], o, *args[1], most, max(lk), workspace=room[:n])
    sta.sta_packed_forward(*args[0], right, *args[1], max(lq), max(lk))
    assert bool((room[n:] == 77).all())
    written = ~torch.isnan(o).any(-1)
    assert bool(written.any()) and float((o.float() - right.float())[written].abs().max()) < 2e-2


def test_keys_beyond_max_k_still_count():
    """max_k only chooses how a launch is cut."""
    q, k, v = randn((2, 4, 64), 1).to(DEV), randn((3000, 1, 64), 2).to(DEV), randn((3000, 1, 64), 3).to(DEV)
    o = [torch.empty_like(q) for _ in range(2)]
    for x, most in zip(o, (3000, 1200)):
        n = sta.sta_packed_workspace_bytes(4, 1, 64, 1, 2, 2, most)
        sta.sta_packed_forward(q, k, v, x, ints([0, 2]), ints([0, 3000]), 2, most, workspace=torch.empty(max(n, 16), dtype=torch.uint8, device=DEV))
    assert float((o[0].double() - o[1].double()).abs().max()) < 2e-3


def test_gradients_against_differences():
    """The loss sum(o g) along random directions, central differences of the definition in 64 bits."""
    Hq, Hkv, D, n = 4, 2, 64, 45
    q, k, v, g = (randn((n, h, D), i + 1) for i, h in enumerate((Hq, Hkv, Hkv, Hq)))
    dev = [x.to(DEV) for x in (q, k, v)]
    o, lse = torch.empty_like(dev[0]), torch.empty((Hq, n), device=DEV)
    cu = ints([0, n])
    sta.sta_packed_forward(*dev, o, cu, cu, n, n, lse=lse)
    d = [torch.empty_like(x) for x in dev]
    ws = torch.empty(sta.sta_packed_backward_workspace_bytes(Hq, n), dtype=torch.uint8, device=DEV)
    sta.sta_packed_backward(*dev, o, g.to(DEV), lse, *d, cu, cu, n, n, ws)

    def loss(q, k, v):
        return float((lu.attention(q, k, v, True, D ** -0.5)[0] * g.double()).sum())

    x = [t.double() for t in (q, k, v)]
    for i in range(3):
        u = torch.randn(x[i].shape, generator=torch.Generator().manual_seed(90 + i), dtype=torch.float64)
        h = 1e-5
        up, down = list(x), list(x)
        up[i], down[i] = x[i] + h * u, x[i] - h * u
        want = (loss(*up) - loss(*down)) / (2 * h)
        got = float((d[i].cpu().double() * u).sum())
        # independent relative errors of up to 2^-7 of the terms add up as their norm; six of those
        assert abs(got - want) <= 6 * 2.0 ** -7 * float((d[i].cpu().double() * u).norm()), (i, got, want)


def test_another_stream_and_a_graph():
    n, Hq, D = 200, 4, 128
    q, k, v = randn((n, Hq, D), 1).to(DEV), randn((n, 2, D), 2).to(DEV), randn((n, 2, D), 3).to(DEV)
    cu, want, o = ints([0, 150, n]), torch.empty_like(q), torch.empty_like(q)
    sta.sta_packed_forward(q, k, v, want, cu, cu, 150, 150)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    sta.sta_packed_forward(q, k, v, o, cu, cu, 150, 150, stream=s)
    s.synchronize()
    assert torch.equal(o, want)
    # single tokens with parts, lengths that change between replays
    q1 = randn((2, Hq, D), 4).to(DEV)
    cu1, cuk, used = ints([0, 1, 2]), ints([0, 2000, 4000]), ints([1900, 7])
    kc, vc = randn((4000, 2, D), 5).to(DEV), randn((4000, 2, D), 6).to(DEV)
    ws = torch.empty(sta.sta_packed_workspace_bytes(Hq, 2, D, 2, 2, 1, 2000), dtype=torch.uint8, device=DEV)
    assert ws.numel() > 0
    y, z = torch.empty_like(q1), torch.empty_like(q1)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        sta.sta_packed_forward(q1, kc, vc, y, cu1, cuk, 1, 2000, k_used=used, workspace=ws)
    for lengths in ([1900, 7], [12, 2000], [0, 1031]):
        used.copy_(torch.tensor(lengths, dtype=torch.int32))
        graph.replay()
        torch.cuda.synchronize()
        sta.sta_packed_forward(q1, kc, vc, z, cu1, cuk, 1, 2000, k_used=used, workspace=torch.empty_like(ws))
        torch.cuda.synchronize()
        assert torch.equal(y, z), lengths


def test_a_cache_beyond_4_gb():
    """Slots whose offsets pass 32 bits give what the same keys give in a small tensor; prompts as well as single tokens."""
    D, Hq, slot, S = 128, 4, 5_400_000, 4
    big = [torch.zeros((S * slot, 1, D), dtype=BF, device=DEV) for _ in range(2)]
    assert big[0].numel() * 2 > 5 * 2 ** 30
    for lq, lk in (([1] * S, [700, 33, 1, 512]), ([70, 1, 33, 140], [700, 33, 65, 512])):
        k, v, q = randn((sum(lk), 1, D), 2).to(DEV), randn((sum(lk), 1, D), 3).to(DEV), randn((sum(lq), Hq, D), 4).to(DEV)
        at = starts(lk)
        for s in range(S):
            for x, y in zip(big, (k, v)):
                x[s * slot:s * slot + lk[s]] = y[at[s]:at[s + 1]]
        want, got = torch.empty_like(q), torch.empty_like(q)
        cu_q, n = ints(starts(lq)), max(lq)
        sta.sta_packed_forward(q, k, v, want, cu_q, ints(at), n, 700)
        sta.sta_packed_forward(q, *big, got, cu_q, ints([s * slot for s in range(S + 1)]), n, 700, k_used=ints(lk))
        assert torch.equal(got, want)
