"""Sizes at which launches of packed sequences end: host side, nothing is launched."""
import pytest

import paper_2502_04507_amd as sta
from paper_2502_04507_amd import layer_ops as lo
from tests import test_packed_refusals as refusals
from tests.test_packed_refusals import ALIAS, M, OK, SHAPE, UNSUPPORTED, WORKSPACE, forward, rows

S24 = 1 << 24


def backward(scale=0.0, **kw):
    if scale == 0.0:
        return refusals.backward(**kw)
    a = dict(S=3, tq=100, tk=300)
    a.update(kw)
    keys = [rows(x * M, 2, 256) for x in (200, 300, 800, 900)]
    return lo._lib().sta_packed_backward(rows(100 * M), keys[0], keys[1], rows(400 * M), rows(450 * M), 600 * M, rows(700 * M), keys[2], keys[3], a["tq"], a["tk"],
                                         500 * M, 501 * M, a["S"], 50, 200, 128, 1, scale, 1000 * M, 1 << 40, None)


@pytest.mark.parametrize("kw", [
    dict(S=S24 // 2, max_q=4), dict(S=S24 // 2, max_q=8),                                   # few rows of 2 key heads: a workgroup each
    dict(S=S24 // 2, max_q=50), dict(S=1 << 30, max_q=1 << 30, max_k=1 << 30),              # tiles
    dict(S=S24, k=rows(200 * M, 1, 128), v=rows(300 * M, 1, 128), max_q=2),
    dict(tq=0x7ffff000 // 8 + 1), dict(tk=0x7ffff001, max_k=200),                           # rows of all heads, and keys, that are counted in 32 bits
])
def test_forward_refuses_launches_of_2_to_the_24_workgroups(kw):
    assert forward(**kw) == SHAPE


@pytest.mark.parametrize("kw", [dict(S=S24 // 2), dict(S=1 << 30), dict(tq=0x7ffff000 // 8 + 1), dict(tk=0x7ffff001)])
def test_gradients_refuse_launches_of_2_to_the_24_workgroups(kw):
    assert backward(nbytes=1 << 40, **kw) == SHAPE


def test_bounds_of_tiles_do_not_overflow():
    # 65,536 heads of one group, as many sequences and as long as 32 bits hold, of one token in all: the products of these pass 64 bits
    f, most = sta.sta_packed_workspace_bytes, 2 ** 31 - 1
    assert f(65536, 1, 64, most, 1, most, most) == 0                                        # more workgroups than a launch has
    assert f(16, 1, 64, 10, 1000, most, 100000) == f(16, 1, 64, 10, 1000, 1000, 100000) > 0  # no sequence is longer than all are together
    # tokens times heads past 64 bits, and past what a call accepts
    assert f(most, 1, 64, 1, 2 ** 62, 1, 100) == f(8, 2, 64, 1, 0x7ffff000 // 8 + 1, 100, 100) == 0
    b = sta.sta_packed_backward_workspace_bytes
    assert b(most, most - 4096) == b(8, 0x7ffff000 // 8 + 1) == 0 and b(8, 0x7ffff000 // 8) > 0
    assert forward(tq=1, tk=100000, S=1, max_q=most, max_k=100000, ws=700 * M, nbytes=f(8, 2, 128, 1, 1, most, 100000) - 1) == WORKSPACE


@pytest.mark.parametrize("batch", [-1, 1 << 41, -(1 << 63)])
def test_the_batch_stride_is_not_looked_at(batch):
    q, k, v, o, g = (rows(*a) for a in ((100 * M,), (200 * M, 2, 256), (300 * M, 2, 256), (400 * M,), (450 * M,)))
    dq, dk, dv = rows(700 * M), rows(800 * M, 2, 256), rows(900 * M, 2, 256)
    for r in (q, k, v, o, g, dq, dk, dv):
        r.batch = batch
    assert forward(q=q, k=k, v=v, o=o, max_q=0) == 0
    assert backward(q=q, k=k, v=v, o=o, d_o=g, dq=dq, dk=dk, dv=dv, S=0) == 0
    assert forward(q=q, k=k, v=v, o=q) == ALIAS             # and does not hide what overlaps
    assert backward(q=q, k=k, v=v, o=o, d_o=g, dq=dq, dk=dk, dv=v) == ALIAS


@pytest.mark.parametrize("scale", [float("nan"), -float("nan"), float("inf"), 2.0 ** 101, 3.0e38])
def test_scales_that_are_no_numbers_or_too_large_are_refused(scale):
    assert forward(scale=scale, max_q=0) == UNSUPPORTED and backward(scale=scale, S=0) == UNSUPPORTED


def test_scales_at_the_ends():
    for scale in (0.0, -0.0, -1.0, -float("inf"), 2.0 ** 100, 2.0 ** -100, 1.0):
        assert forward(scale=scale, max_q=0) == OK and backward(scale=scale, S=0) == OK
    for scale in (2.0 ** -101, 1e-38, 1e-44):                # gradients divide by it
        assert forward(scale=scale, max_q=0) == OK and backward(scale=scale, S=0) == UNSUPPORTED


@pytest.mark.parametrize("kw", [
    dict(cu_q=400 * M + 1024), dict(cu_k=400 * M), dict(used=400 * M + 100 * 2048 - 4), dict(cu_q=600 * M + 64, lse=600 * M), dict(used=600 * M + 3196, lse=600 * M),
    dict(cu_k=600 * M - 12, lse=600 * M), dict(cu_k=700 * M + 4, ws=700 * M, nbytes=1 << 20), dict(used=700 * M - 8, ws=700 * M, nbytes=1 << 20),
])
def test_forward_refuses_to_write_its_bounds(kw):
    assert forward(**kw) == ALIAS


@pytest.mark.parametrize("kw", [dict(cu_q=700 * M), dict(cu_k=700 * M + 2048), dict(cu_q=800 * M - 12), dict(cu_k=900 * M + 4), dict(cu_q=1000 * M + 8), dict(cu_k=1000 * M - 4)])
def test_gradients_refuse_to_write_their_bounds(kw):
    assert refusals.backward(**kw) == ALIAS
