"""Which tensors of rows the argument checks take to overlap, against the sets of their bytes (host side, nothing is launched)."""
import ctypes
import random

import pytest

import paper_2502_04507_amd as sta
from paper_2502_04507_amd import layer_ops as lo

M = 1 << 20


def overlap(a, Na, b, Nb, B, D):
    fn = sta.load_library().sta_rows_overlap
    fn.argtypes = [ctypes.POINTER(lo._HeadRows), ctypes.c_int64] * 2 + [ctypes.c_int64, ctypes.c_int]
    return bool(fn(a, Na, b, Nb, B, D))


def touched(r, B, N, D):
    size = 4 if r.dtype else 2
    starts = {r.data + size * (b * r.batch + n * r.token + h * r.head) for b in range(B) for n in range(N) for h in range(r.heads)}
    return {s + x for s in starts for x in range(D * size)}


def test_small_tensors_of_any_strides():
    rng = random.Random(5)
    verdicts = {True: 0, False: 0}
    for _ in range(6000):
        B, D, n = rng.choice([1, 1, 2, 3]), rng.choice([1, 2, 5]), [rng.choice([1, 2, 3, 4]) for _ in range(2)]
        make = [lo._HeadRows(M + 2 * rng.randrange(0, 80), rng.randrange(0, 60), rng.randrange(0, 25), rng.randrange(0, 25), rng.choice([1, 2, 3]), rng.choice([0, 0, 1]))
                for _ in range(2)]
        if rng.random() < 0.5:                              # the strides alike, as of views of one tensor
            for field in rng.sample(["batch", "token", "head", "dtype"], rng.randrange(1, 5)):
                setattr(make[1], field, getattr(make[0], field))
        want = bool(touched(make[0], B, n[0], D) & touched(make[1], B, n[1], D))
        assert overlap(make[0], n[0], make[1], n[1], B, D) == want, [(r.data, r.batch, r.token, r.head, r.heads, r.dtype) for r in make] + [B, n, D]
        verdicts[want] += 1
    assert min(verdicts.values()) > 1000


def rows(data, batch, token, head, heads, dtype=0):
    return lo._HeadRows(data, batch, token, head, heads, dtype)


@pytest.mark.parametrize("B,N,C,Hq,Hkv,D,pad", [(2, 33, 64, 8, 2, 128, 0), (3, 115200, 115200, 24, 24, 128, 0), (2, 1, 4096, 32, 8, 128, 24), (5, 700, 701, 3, 1, 80, 7)])
def test_views_side_by_side_do_not_overlap(B, N, C, Hq, Hkv, D, pad):
    H = Hq + 2 * Hkv
    layouts = {
        # head ranges of one [B, Hq + 2 Hkv, N, D]
        "head-major": [rows(M + 2 * first * N * D, H * N * D, D, N * D, h) for first, h in ((0, Hq), (Hq, Hkv), (Hq + Hkv, Hkv))],
        # keys and values in one cache [B, 2, Hkv, C, D]
        "cache": [rows(M + 2 * i * Hkv * C * D, 2 * Hkv * C * D, D, C * D, Hkv) for i in range(2)],
        # one [B, N, Hq + 2 Hkv, D] whose batch stride is no multiple of the token stride
        "token-major": [rows(M + 2 * first * D, N * H * D + pad, H * D, D, h) for first, h in ((0, Hq), (Hq, Hkv), (Hq + Hkv, Hkv))],
        # channels of one row [B, N, H, 3 D]
        "channels": [rows(M + 2 * i * D, N * Hq * 3 * D + pad, Hq * 3 * D, 3 * D, Hq) for i in range(3)],
        # every third token of one [B, 3 N, Hkv, D]
        "tokens in turn": [rows(M + 2 * i * Hkv * D, 3 * N * Hkv * D, 3 * Hkv * D, D, Hkv) for i in range(3)],
    }
    for name, views in layouts.items():
        for i, a in enumerate(views):
            for j, b in enumerate(views):
                assert overlap(a, N, b, N, B, D) == (i == j), (name, i, j)
        if name == "cache" and C > N:                       # (tokens that are not written lie between)
            continue
        for a, b in zip(views, views[1:]):                  # an element further reaches into the neighbour
            assert overlap(rows(a.data + 2, a.batch, a.token, a.head, a.heads), N, b, N, B, D), name
