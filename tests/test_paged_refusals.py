"""What the operators on a cache in pages refuse: host side, nothing is launched."""
import pytest
import torch

import paper_2502_04507_amd as sta
from paper_2502_04507_amd import layer_ops as lo
from paper_2502_04507_amd import paged_ops as po

OK, NULL, SHAPE, UNSUPPORTED, ALIAS, WORKSPACE = 0, 1, 2, 4, 5, 6
M = 1 << 20


def rows(data, heads=8, token=1024, head=128, dtype=0, batch=0):
    return lo._HeadRows(data, batch, token, head, heads, dtype)


def pool(data, heads=2, page=4096, token=256, head=128, dtype=0):
    return rows(data, heads, token, head, dtype, page)


def cache(**kw):
    a = dict(k=pool(200 * M), v=pool(300 * M), pages=1000, page_size=16, table=500 * M, row=40, width=40, used=501 * M)
    a.update(kw)
    return po._PagedCache(a["k"], a["v"], a["pages"], a["page_size"], a["table"], a["row"], a["width"], a["used"])


def both(**kw):
    """Of k and v of a cache alike."""
    return cache(k=pool(200 * M, **kw), v=pool(300 * M, **kw))


def forward(**kw):
    a = dict(q=rows(100 * M), o=rows(400 * M), lse=None, tq=100, cu=502 * M, cache=cache(), S=3, max_q=50, max_k=200, D=128, scale=0.0, ws=None, nbytes=0)
    a.update(kw)
    return po._lib().sta_paged_forward(a["q"], a["o"], a["lse"], a["tq"], a["cu"], a["cache"], a["S"], a["max_q"], a["max_k"], a["D"], 1, a["scale"], a["ws"],
                                       a["nbytes"], None)


# what every entry refuses of a cache
CACHES = [
    (NULL, dict(cache=None)), (NULL, dict(cache=cache(k=pool(None)))), (NULL, dict(cache=cache(table=None))), (NULL, dict(cache=cache(used=None))),
    (SHAPE, dict(cache=cache(pages=-1))), (SHAPE, dict(cache=cache(pages=1 << 31))), (SHAPE, dict(cache=cache(page_size=0))), (SHAPE, dict(cache=cache(width=-1))),
    (SHAPE, dict(cache=cache(row=-1))), (SHAPE, dict(cache=cache(row=1 << 41))), (SHAPE, dict(cache=cache(table=500 * M + 2))), (SHAPE, dict(cache=cache(used=500 * M + 1))),
    (SHAPE, dict(cache=cache(k=pool(200 * M + 8)))), (SHAPE, dict(cache=cache(v=pool(300 * M, page=8192)))), (SHAPE, dict(cache=cache(v=pool(300 * M, heads=1)))),
    (SHAPE, dict(cache=both(token=260))), (SHAPE, dict(cache=both(head=132))), (SHAPE, dict(cache=both(page=4100))), (SHAPE, dict(cache=both(page=1 << 31))),
    (SHAPE, dict(cache=both(token=1 << 27))), (SHAPE, dict(cache=both(page=256, token=1 << 26))), (UNSUPPORTED, dict(cache=both(dtype=1))), (SHAPE, dict(S=-1)), (UNSUPPORTED, dict(D=96)),
]


@pytest.mark.parametrize("want,kw", CACHES + [
    (NULL, dict(q=None)), (NULL, dict(o=rows(None))), (NULL, dict(cu=None)), (SHAPE, dict(tq=-1)), (SHAPE, dict(max_k=-2)), (SHAPE, dict(tq=1 << 31)),
    (UNSUPPORTED, dict(q=rows(100 * M, dtype=1))), (UNSUPPORTED, dict(scale=float("nan"))), (UNSUPPORTED, dict(scale=2.0 ** 101)), (SHAPE, dict(q=rows(100 * M + 8))),
    (SHAPE, dict(o=rows(400 * M, 7))), (SHAPE, dict(q=rows(100 * M, 7), o=rows(400 * M, 7))), (SHAPE, dict(cu=502 * M + 2)), (SHAPE, dict(lse=600 * M + 1)),
    (SHAPE, dict(S=1 << 23, max_q=4)), (ALIAS, dict(o=rows(100 * M))), (ALIAS, dict(o=rows(200 * M))), (ALIAS, dict(o=rows(300 * M + 4096))), (ALIAS, dict(lse=400 * M)),
    (ALIAS, dict(lse=300 * M + 64)), (ALIAS, dict(lse=500 * M)), (ALIAS, dict(lse=501 * M + 8)), (ALIAS, dict(lse=502 * M)), (ALIAS, dict(o=rows(502 * M - 1024))),
    (WORKSPACE, dict(ws=700 * M + 8, nbytes=1 << 30)), (ALIAS, dict(ws=100 * M, nbytes=1 << 20)), (ALIAS, dict(ws=500 * M - 64, nbytes=1 << 10)),
    (ALIAS, dict(ws=600 * M, nbytes=1 << 20, lse=600 * M + 1024)), (ALIAS, dict(ws=200 * M, nbytes=16)), (OK, dict(S=0)), (OK, dict(tq=0)), (OK, dict(max_q=0)),
    (OK, dict(S=0, cache=cache(table=None, used=None))), (OK, dict(max_q=0, cache=cache(k=pool(None), v=pool(None), pages=0))),
])
def test_forward_refuses(want, kw):
    assert forward(**kw) == want


def test_forward_refuses_a_small_workspace():
    need = sta.sta_paged_workspace_bytes(8, 2, 128, 1, 1, 1, 100000)
    assert need == sta.sta_packed_workspace_bytes(8, 2, 128, 1, 1, 1, 100000) > 0
    kw = dict(tq=1, S=1, max_q=1, max_k=100000, ws=700 * M)
    assert forward(nbytes=need - 1, **kw) == WORKSPACE


def append(**kw):
    a = dict(k=rows(100 * M, 2), v=rows(110 * M, 2), tq=100, cu=502 * M, cache=cache(), S=3, max_new=50, D=128, weights=None)
    a.update(kw)
    return po._lib().sta_paged_append(a["k"], a["v"], a["tq"], a["cu"], a["cache"], a["S"], a["max_new"], a["D"], a["weights"], None)


@pytest.mark.parametrize("want,kw", CACHES + [
    (NULL, dict(k=None)), (NULL, dict(v=rows(None, 2))), (NULL, dict(cu=None)), (SHAPE, dict(tq=-1)), (SHAPE, dict(max_new=-1)), (SHAPE, dict(tq=1 << 31)), (SHAPE, dict(S=65536)),
    (SHAPE, dict(k=rows(100 * M, 3))), (SHAPE, dict(v=rows(110 * M + 8, 2))), (SHAPE, dict(k=rows(100 * M, 2, token=260))), (SHAPE, dict(v=rows(110 * M, 2, head=132))),
    (UNSUPPORTED, dict(k=rows(100 * M, 2, dtype=1))), (UNSUPPORTED, dict(k=rows(100 * M, 2, dtype=2))), (SHAPE, dict(k=rows(100 * M, 2, token=262, dtype=1), v=rows(110 * M, 2, dtype=1))),
    (SHAPE, dict(cu=502 * M + 1)), (SHAPE, dict(weights=600 * M + 2)),
    # a pool whose pages, slots or heads lie in each other, or keys among values
    (SHAPE, dict(cache=both(page=2048))), (SHAPE, dict(cache=both(token=128))), (SHAPE, dict(cache=both(head=64))), (ALIAS, dict(cache=cache(v=pool(200 * M)))),
    (ALIAS, dict(cache=cache(v=pool(200 * M + 16)))),
    (ALIAS, dict(k=rows(200 * M, 2))), (ALIAS, dict(v=rows(300 * M + 8192, 2))), (ALIAS, dict(weights=200 * M)), (ALIAS, dict(weights=300 * M + 64)), (ALIAS, dict(weights=100 * M)),
    (ALIAS, dict(weights=110 * M + 64)), (ALIAS, dict(weights=500 * M)), (ALIAS, dict(weights=501 * M)), (ALIAS, dict(weights=502 * M)), (ALIAS, dict(cu=200 * M + 64)),
    (ALIAS, dict(cache=cache(table=300 * M))), (ALIAS, dict(cache=cache(used=200 * M))),
    (OK, dict(S=0)), (OK, dict(tq=0)), (OK, dict(max_new=0)), (OK, dict(cache=cache(width=0, table=None))), (OK, dict(cache=cache(pages=0, k=pool(None), v=pool(None)))),
])
def test_append_refuses(want, kw):
    assert append(**kw) == want


def weights(**kw):
    a = dict(q=rows(100 * M), lse=600 * M, tq=100, cu=502 * M, cache=cache(), S=3, max_q=50, max_k=200, D=128, scale=0.0, before=None, decay=1.0, weights=700 * M)
    a.update(kw)
    return po._lib().sta_paged_weights(a["q"], a["lse"], a["tq"], a["cu"], a["cache"], a["S"], a["max_q"], a["max_k"], a["D"], 1, a["scale"], a["before"], a["decay"],
                                       a["weights"], None)


@pytest.mark.parametrize("want,kw", CACHES + [
    (NULL, dict(q=None)), (NULL, dict(lse=None)), (NULL, dict(weights=None)), (NULL, dict(cu=None)), (SHAPE, dict(tq=-1)), (SHAPE, dict(max_q=-1)), (SHAPE, dict(max_k=-1)),
    (SHAPE, dict(tq=1 << 31)), (UNSUPPORTED, dict(q=rows(100 * M, dtype=1))), (UNSUPPORTED, dict(scale=float("nan"))), (UNSUPPORTED, dict(decay=float("nan"))),
    (UNSUPPORTED, dict(decay=float("inf"))), (UNSUPPORTED, dict(decay=-float("inf"))), (SHAPE, dict(q=rows(100 * M, 7))), (SHAPE, dict(q=rows(100 * M + 4))),
    (SHAPE, dict(cu=502 * M + 2)), (SHAPE, dict(lse=600 * M + 1)), (SHAPE, dict(weights=700 * M + 2)), (SHAPE, dict(before=800 * M + 2)),
    (SHAPE, dict(S=1 << 24, max_k=64)), (SHAPE, dict(S=1 << 16, max_k=1 << 30, cache=cache(width=1 << 26, row=1 << 26))),
    (ALIAS, dict(weights=100 * M)), (ALIAS, dict(weights=200 * M)), (ALIAS, dict(weights=300 * M + 4)), (ALIAS, dict(weights=500 * M)), (ALIAS, dict(weights=501 * M)),
    (ALIAS, dict(weights=502 * M)), (ALIAS, dict(weights=600 * M)), (ALIAS, dict(before=700 * M + 4)), (ALIAS, dict(before=700 * M - 4)),
    (OK, dict(S=0)), (OK, dict(max_k=0)), (OK, dict(cache=cache(width=0, table=None))), (OK, dict(cache=cache(pages=0, k=pool(None), v=pool(None)))),
])
def test_weights_refuses(want, kw):
    assert weights(**kw) == want


def into(**kw):
    a = dict(k=pool(1200 * M), v=pool(1300 * M), pages=500, table=1500 * M, used=1501 * M)
    a.update(kw)
    return cache(**a)


def evict(**kw):
    a = dict(cache=cache(), weights=700 * M, into=into(), into_weights=1700 * M, kept=1800 * M, S=3, keep=128, first=4, recent=32, D=128)
    a.update(kw)
    return po._lib().sta_paged_evict(a["cache"], a["weights"], a["into"], a["into_weights"], a["kept"], a["S"], a["keep"], a["first"], a["recent"], a["D"], None)


@pytest.mark.parametrize("want,kw", CACHES + [
    (NULL, dict(into=None)), (NULL, dict(weights=None)), (NULL, dict(kept=None)), (NULL, dict(into=into(used=None))), (NULL, dict(into=into(table=None))),
    (SHAPE, dict(keep=-1)), (SHAPE, dict(first=-1)), (SHAPE, dict(recent=-1)), (SHAPE, dict(first=100, recent=29)), (SHAPE, dict(first=2 ** 31 - 1, recent=2 ** 31 - 1)),
    (SHAPE, dict(into=into(k=pool(1200 * M, 1), v=pool(1300 * M, 1)))), (SHAPE, dict(into=into(width=7))), (SHAPE, dict(keep=641)), (SHAPE, dict(S=1 << 21)),
    (SHAPE, dict(S=1 << 20, keep=640)), (SHAPE, dict(into=into(k=pool(1200 * M, page=2048), v=pool(1300 * M, page=2048)))), (SHAPE, dict(weights=700 * M + 1)),
    (SHAPE, dict(into_weights=1700 * M + 2)), (SHAPE, dict(kept=1800 * M + 2)),
    # pools that share memory without being the same
    (ALIAS, dict(into=into(k=pool(200 * M + 4096)))), (ALIAS, dict(into=into(v=pool(200 * M)))), (ALIAS, dict(into=into(k=pool(300 * M)))), (ALIAS, dict(into=into(k=pool(200 * M)))),
    (ALIAS, dict(into=into(v=pool(1200 * M)))), (ALIAS, dict(into_weights=700 * M)), (ALIAS, dict(into_weights=700 * M + 4)), (ALIAS, dict(into_weights=200 * M)),
    (ALIAS, dict(into_weights=1300 * M)), (ALIAS, dict(into_weights=500 * M)), (ALIAS, dict(into_weights=1500 * M)), (ALIAS, dict(into_weights=1501 * M)),
    (ALIAS, dict(into_weights=1800 * M)), (ALIAS, dict(kept=700 * M)), (ALIAS, dict(kept=1700 * M)), (ALIAS, dict(kept=1200 * M)), (ALIAS, dict(kept=300 * M)),
    (ALIAS, dict(kept=500 * M)), (ALIAS, dict(kept=501 * M)), (ALIAS, dict(kept=1500 * M)), (ALIAS, dict(kept=1501 * M)), (ALIAS, dict(into=into(used=501 * M))),
    (ALIAS, dict(into=into(used=1500 * M))), (ALIAS, dict(into=into(used=700 * M))), (ALIAS, dict(into=into(used=200 * M))), (ALIAS, dict(into=into(used=1300 * M))),
    (ALIAS, dict(into=into(k=pool(500 * M - 64)))), (ALIAS, dict(into=into(v=pool(700 * M)))), (ALIAS, dict(into=into(table=1200 * M))), (OK, dict(S=0)),
])
def test_evict_refuses(want, kw):
    assert evict(**kw) == want


def test_keys_and_values_of_a_page_side_by_side_do_not_overlap():
    # [pages, 2, slots, heads, D] and [pages, slots, 2, heads, D]; max_new 0, as anything else would be launched
    for apart, page, token in ((4096, 8192, 256), (256, 8192, 512)):
        c = cache(k=pool(200 * M, page=page, token=token), v=pool(200 * M + 2 * apart, page=page, token=token))
        assert append(cache=c, max_new=0) == OK
        assert append(cache=c, weights=200 * M + 64) == ALIAS


def test_the_class_refuses():
    k, t, u = torch.zeros((4, 16, 2, 64), dtype=torch.bfloat16), torch.zeros((3, 5), dtype=torch.int32), torch.zeros(3, dtype=torch.int32)
    for args, match in (
        ((k.float(), k, t, u), "bfloat16"), ((k[0], k[0], t, u), "pages"), ((k, k[:2], t, u), "pages"), ((k, k.transpose(1, 2).contiguous().transpose(1, 2), t, u), "laid out alike"),
        ((k, k, t.long(), u), "table must be int32"), ((k, k, t[0], u), "table"), ((k, k, t.t()[:3], u), "adjacent"), ((k, k, t, u[:2]), "used must be"), ((k, k, t, u.long()), "used must be"),
        ((k, k, t, u), "device memory"),
    ):
        with pytest.raises(ValueError, match=match):
            sta.StaPagedCache(*args)


@pytest.mark.parametrize("name", ["k", "v", "table", "used", "room"])
def test_a_cache_keeps_its_tensors(name):
    """Calls take addresses that were looked up when the cache was made: another tensor in an attribute's place would not be seen."""
    with pytest.raises(AttributeError):
        setattr(object.__new__(sta.StaPagedCache), name, None)
