"""What attention over packed sequences refuses: host side, nothing is launched."""
import pytest

import paper_2502_04507_amd as sta
from paper_2502_04507_amd import layer_ops as lo

OK, NULL, SHAPE, UNSUPPORTED, ALIAS, WORKSPACE = 0, 1, 2, 4, 5, 6
M = 1 << 20


def rows(data, heads=8, token=1024, head=128, dtype=0):
    return lo._HeadRows(data, 0, token, head, heads, dtype)


def forward(**kw):
    a = dict(q=rows(100 * M), k=rows(200 * M, 2, 256), v=rows(300 * M, 2, 256), o=rows(400 * M), lse=None, tq=100, tk=300, cu_q=500 * M, cu_k=501 * M,
             used=None, S=3, max_q=50, max_k=200, D=128, causal=1, scale=0.0, ws=None, nbytes=0)
    a.update(kw)
    return lo._lib().sta_packed_forward(a["q"], a["k"], a["v"], a["o"], a["lse"], a["tq"], a["tk"], a["cu_q"], a["cu_k"], a["used"], a["S"], a["max_q"],
                                        a["max_k"], a["D"], a["causal"], a["scale"], a["ws"], a["nbytes"], None)


@pytest.mark.parametrize("want,kw", [
    (NULL, dict(q=None)), (NULL, dict(o=rows(None))), (NULL, dict(cu_q=None)), (NULL, dict(cu_k=None)), (SHAPE, dict(S=-1)), (SHAPE, dict(tq=-1)), (SHAPE, dict(max_k=-2)),
    (SHAPE, dict(tq=1 << 31)), (SHAPE, dict(tk=1 << 31)), (UNSUPPORTED, dict(D=96)), (UNSUPPORTED, dict(q=rows(100 * M, dtype=1))), (SHAPE, dict(q=rows(100 * M + 8))),
    (SHAPE, dict(k=rows(200 * M, 2, 260))), (SHAPE, dict(v=rows(300 * M, 2, 256, 132))), (SHAPE, dict(v=rows(300 * M, 1, 256))), (SHAPE, dict(k=rows(200 * M, 3, 512), v=rows(300 * M, 3, 512))),
    (SHAPE, dict(o=rows(400 * M, 7))), (SHAPE, dict(o=rows(400 * M, token=512))), (SHAPE, dict(q=rows(100 * M, token=1 << 26))), (SHAPE, dict(cu_q=500 * M + 2)), (SHAPE, dict(lse=600 * M + 1)),
    (ALIAS, dict(o=rows(100 * M))), (ALIAS, dict(o=rows(200 * M))), (ALIAS, dict(lse=400 * M)), (ALIAS, dict(lse=300 * M + 64)), (WORKSPACE, dict(ws=700 * M + 8, nbytes=1 << 30)),
    (ALIAS, dict(ws=100 * M, nbytes=1 << 20)), (ALIAS, dict(ws=600 * M, nbytes=1 << 20, lse=600 * M + 1024)), (OK, dict(S=0)), (OK, dict(tq=0)), (OK, dict(max_q=0)),
])
def test_forward_refuses(want, kw):
    assert forward(**kw) == want


def test_forward_refuses_a_small_workspace():
    need = sta.sta_packed_workspace_bytes(8, 2, 128, 1, 1, 1, 100000)
    assert need > 0
    kw = dict(tq=1, tk=100000, S=1, max_q=1, max_k=100000, ws=700 * M)
    assert forward(nbytes=need - 1, **kw) == WORKSPACE


def backward(**kw):
    a = dict(q=rows(100 * M), k=rows(200 * M, 2, 256), v=rows(300 * M, 2, 256), o=rows(400 * M), d_o=rows(450 * M), lse=600 * M, dq=rows(700 * M),
             dk=rows(800 * M, 2, 256), dv=rows(900 * M, 2, 256), tq=100, tk=300, cu_q=500 * M, cu_k=501 * M, S=3, D=128, ws=1000 * M,
             nbytes=sta.sta_packed_backward_workspace_bytes(8, 100))
    a.update(kw)
    return lo._lib().sta_packed_backward(a["q"], a["k"], a["v"], a["o"], a["d_o"], a["lse"], a["dq"], a["dk"], a["dv"], a["tq"], a["tk"], a["cu_q"], a["cu_k"],
                                         a["S"], 50, 200, a["D"], 1, 0.0, a["ws"], a["nbytes"], None)


@pytest.mark.parametrize("want,kw", [
    (NULL, dict(lse=None)), (NULL, dict(dk=None)), (NULL, dict(cu_k=None)), (SHAPE, dict(S=-1)), (UNSUPPORTED, dict(D=32)), (UNSUPPORTED, dict(dv=rows(900 * M, 2, 256, dtype=1))),
    (SHAPE, dict(dq=rows(700 * M, 4))), (SHAPE, dict(dk=rows(800 * M, 2, 128))), (SHAPE, dict(d_o=rows(450 * M + 2))), (SHAPE, dict(lse=600 * M + 2)), (WORKSPACE, dict(ws=None)),
    (WORKSPACE, dict(nbytes=1000)), (WORKSPACE, dict(ws=1000 * M + 4)), (ALIAS, dict(dq=rows(100 * M))), (ALIAS, dict(dv=rows(800 * M, 2, 256))), (ALIAS, dict(dk=rows(450 * M, 2, 256))),
    (ALIAS, dict(ws=600 * M)), (ALIAS, dict(ws=900 * M)), (ALIAS, dict(ws=100 * M)), (ALIAS, dict(lse=700 * M)), (OK, dict(S=0)), (OK, dict(tq=0, tk=0)),
])
def test_backward_refuses(want, kw):
    assert backward(**kw) == want


def test_tensors_without_tokens_need_no_memory_and_meet_nothing():
    none, keys = rows(None), rows(None, 2, 256)
    assert forward(q=none, o=none, tq=0) == OK
    assert backward(q=none, k=keys, v=keys, o=none, d_o=none, lse=None, dq=none, dk=keys, dv=keys, tq=0, tk=0) == OK
    same = rows(100 * M, 2, 256)                # where nothing is, nothing overlaps; what is there still does
    assert forward(k=same, v=same, tk=0, o=rows(100 * M)) == ALIAS
    assert backward(k=same, v=same, dk=same, dv=same, tk=0, dq=rows(100 * M)) == ALIAS
    assert forward(k=rows(None, 2, 256), tk=0, tq=1 << 31) == SHAPE
    assert forward(k=keys, v=keys, tk=1) == NULL


def test_workspace_bytes():
    f, b = sta.sta_packed_workspace_bytes, sta.sta_packed_backward_workspace_bytes
    assert f(8, 3, 128, 1, 1, 1, 100) == f(8, 2, 96, 1, 1, 1, 100) == f(8, 2, 128, -1, 1, 1, 100) == f(0, 1, 64, 1, 1, 1, 100) == 0
    assert f(32, 8, 128, 64, 64 * 4096, 4096, 4096) == 0            # fills the chip uncut
    assert b(0, 5) == b(4, -1) == 0 and b(4, 1000) >= 2 * 4 * 1000 * 4
