"""What the row operators refuse, and the steps of rotary positions: host side, nothing is launched."""
import ctypes
import math

import pytest

import paper_2502_04507_amd as sta
from paper_2502_04507_amd import layer_ops as lo

OK, NULL, SHAPE, UNSUPPORTED, ALIAS, WORKSPACE = 0, 1, 2, 4, 5, 6


def rows(data=1 << 20, batch=4096, token=512, head=128, heads=4, dtype=0):
    return lo._HeadRows(data, batch, token, head, heads, dtype)


def rotary(steps=1 << 40, positions=None, channels=128, pairs=(64, 0, 0), **kw):
    r = lo._Rotary(steps, positions, 0, 1, channels, (ctypes.c_int * 3)(*pairs), 0, 1.0)
    for k, v in kw.items():
        setattr(r, k, v)
    return r


def rope(x=None, out=None, n=1, B=2, N=8, D=128, rot=None):
    return lo._lib().sta_rope(x or rows(), out or rows(1 << 30), n, B, N, D, rot or rotary(), 0, None)


@pytest.mark.parametrize("want,kw", [
    (NULL, dict(x=rows(data=None))), (NULL, dict(rot=rotary(steps=None))), (SHAPE, dict(n=0)), (SHAPE, dict(n=4)), (SHAPE, dict(B=-1)),
    (UNSUPPORTED, dict(D=0)), (UNSUPPORTED, dict(D=127)), (UNSUPPORTED, dict(D=258)), (SHAPE, dict(B=1 << 16, N=1 << 16)),
    (SHAPE, dict(rot=rotary(channels=130, pairs=(65, 0, 0)))), (SHAPE, dict(rot=rotary(channels=127))), (SHAPE, dict(rot=rotary(pairs=(60, 0, 0)))),
    (SHAPE, dict(rot=rotary(pairs=(70, -6, 0)))), (SHAPE, dict(rot=rotary(pairs=(32, 16, 16)))), (SHAPE, dict(rot=rotary(steps=(1 << 40) + 4))),
    (SHAPE, dict(rot=rotary(positions=(1 << 30) + 2))), (SHAPE, dict(rot=rotary(position_token=-1))),
    (UNSUPPORTED, dict(x=rows(dtype=2))), (SHAPE, dict(x=rows(data=(1 << 20) + 1))), (SHAPE, dict(x=rows(heads=0))), (SHAPE, dict(x=rows(token=-512))),
    (SHAPE, dict(out=rows(1 << 30, heads=3))), (SHAPE, dict(out=rows(1 << 30, token=0))), (SHAPE, dict(out=rows(1 << 30, head=64))),
    (SHAPE, dict(out=rows(1 << 30, token=500))), (ALIAS, dict(out=rows((1 << 20) + 256))), (ALIAS, dict(out=rows(dtype=1))),
    (ALIAS, dict(out=rows(1 << 20, token=1024, batch=8192))), (OK, dict(N=0)), (OK, dict(B=0)),
])
def test_rope_refuses(want, kw):
    assert rope(**kw) == want


def test_fused_heads_do_not_alias_but_shifted_ones_do():
    # queries at heads 0..3 and keys at 4..5 of rows of 6 heads: in place on both is no overlap; a shift by one head is
    a = (lo._HeadRows * 2)(rows(heads=4, token=768, batch=8 * 768), rows((1 << 20) + 4 * 256, heads=2, token=768, batch=8 * 768))
    shifted = (lo._HeadRows * 2)(a[0], rows((1 << 20) + 3 * 256, heads=2, token=768, batch=8 * 768))
    assert lo._lib().sta_rope(a, shifted, 2, 2, 8, 128, rotary(), 0, None) == ALIAS
    assert lo._lib().sta_rope(a, a, 2, 0, 8, 128, rotary(), 0, None) == OK


def norm(q=None, v=None, v_out=None, grid=None, tile=None, weight_dt=1, N=8, D=128, rot=None, wq=1 << 41):
    i3 = ctypes.c_int * 3
    return lo._lib().sta_qk_norm_rope(q or rows(), rows(1 << 25), v, rows(1 << 30), rows(1 << 31), v_out, wq, None, weight_dt, 1e-6,
                                      rot, 2, N, D, None if grid is None else i3(*grid), None if tile is None else i3(*tile), None)


@pytest.mark.parametrize("want,kw", [
    (NULL, dict(q=rows(data=None))), (NULL, dict(v=rows(1 << 26))), (NULL, dict(tile=(1, 1, 1))), (SHAPE, dict(grid=(1, 2, 5))), (SHAPE, dict(grid=(1, 2, 4), tile=(1, 2, 3))),
    (SHAPE, dict(grid=(1, 0, 4))), (UNSUPPORTED, dict(weight_dt=7)), (SHAPE, dict(wq=(1 << 41) + 2)), (UNSUPPORTED, dict(D=300)),
    (ALIAS, dict(q=rows(1 << 30), grid=(1, 2, 4), tile=(1, 2, 2))), (OK, dict(N=0)),
])
def test_norm_rope_refuses(want, kw):
    assert norm(**kw) == want


@pytest.mark.parametrize("want,kw", [
    (WORKSPACE, dict(ws=None)), (WORKSPACE, dict(nbytes=100)), (WORKSPACE, dict(ws=(1 << 42) + 8)), (ALIAS, dict(ws=1 << 20)), (ALIAS, dict(dq=1 << 20)),
    (ALIAS, dict(dq=1 << 27)), (SHAPE, dict(dw=(1 << 43) + 2)), (NULL, dict(dq=None)),
])
def test_norm_rope_backward_refuses(want, kw):
    a = dict(ws=1 << 42, nbytes=sta.sta_qk_norm_rope_workspace_bytes(128), dq=1 << 30, dw=1 << 43)
    a.update(kw)
    got = lo._lib().sta_qk_norm_rope_backward(rows(), rows(1 << 25), rows(1 << 27), rows(1 << 28), None, rows(a["dq"]), rows(1 << 31), None, None,
                                              None, 1, a["dw"], None, 1e-6, None, 2, 8, 128, None, None, a["ws"], a["nbytes"], None)
    assert got == want


def test_norm_rope_refuses_weights_inside_an_output():
    assert norm(wq=(1 << 30) + 512) == ALIAS
    assert norm(wq=(1 << 31) + 1024) == ALIAS


@pytest.mark.parametrize("kw", [
    dict(dw=(1 << 42) + 64), dict(dw=1 << 20), dict(dw=1 << 27), dict(dw=(1 << 30) + 256), dict(dw=1 << 44, dw2=(1 << 44) + 256), dict(dw=(1 << 45) + 256),
    dict(wq=(1 << 30) + 256), dict(dw2=1 << 31),
])
def test_norm_rope_backward_refuses_weight_gradients_inside_what_it_uses(kw):
    a = dict(ws=1 << 42, dw=1 << 43, dw2=None, wq=1 << 45)
    a.update(kw)
    assert lo._lib().sta_qk_norm_rope_backward(rows(), rows(1 << 25), rows(1 << 27), rows(1 << 28), None, rows(1 << 30), rows(1 << 31), None, a["wq"],
                                               None, 1, a["dw"], a["dw2"], 1e-6, None, 2, 8, 128, None, None, a["ws"],
                                               sta.sta_qk_norm_rope_workspace_bytes(128), None) == ALIAS


def test_workspace_bytes():
    assert sta.sta_qk_norm_rope_workspace_bytes(128) > 0
    assert sta.sta_qk_norm_rope_workspace_bytes(0) == sta.sta_qk_norm_rope_workspace_bytes(129) == sta.sta_qk_norm_rope_workspace_bytes(258) == 0


def _turns(f):
    return round(f / (2 * math.pi) * 2.0 ** 64)


@pytest.mark.parametrize("channels,theta", [(2, 10000.0), (64, 10000.0), (128, 500000.0), (56, 256.0)])
def test_rope_steps(channels, theta):
    pairs = channels // 2
    plain = [theta ** (-2.0 * i / channels) for i in range(pairs)]
    ntk_theta = theta * 4.0 ** (channels / (channels - 2.0)) if pairs > 1 else theta
    yarn = []
    for f in plain:
        k = min(1.0, max(0.0, (2048 * f / (2 * math.pi) - 1.0) / 31.0))
        yarn.append(f * (1 - k) / 4.0 + f * k)
    for scaling, want, magnitude in ((sta.STA_ROPE_NONE, plain, 1.0), (sta.STA_ROPE_LINEAR, [f / 4.0 for f in plain], 1.0),
                                     (sta.STA_ROPE_NTK, [ntk_theta ** (-2.0 * i / channels) for i in range(pairs)], 1.0),
                                     (sta.STA_ROPE_YARN, yarn, 0.1 * math.log(4.0) + 1.0)):
        steps, m = sta.sta_rope_steps(channels, theta, scaling, 4.0, 2048)
        assert abs(m - magnitude) < 1e-6
        for got, f in zip(steps.tolist(), want):
            assert abs(got - _turns(f)) <= 1e-13 * _turns(f) + 1


@pytest.mark.parametrize("args", [(0,), (3,), (258,), (64, 0.5), (64, float("nan")), (64, 1e4, 9), (64, 1e4, 1, 0.5), (64, 1e4, 3, 2.0, 0.0)])
def test_rope_steps_refuses(args):
    with pytest.raises(sta.StaError):
        sta.sta_rope_steps(*args)
