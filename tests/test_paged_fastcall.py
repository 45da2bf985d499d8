"""The operators on a cache in pages through the extension and through ctypes: the same results, the same errors, and everything that the extension does not know is
left to the general path."""
import pytest
import torch

import paper_2502_04507_amd as sta
from paper_2502_04507_amd import binding

BF = torch.bfloat16


def test_leaves_what_it_does_not_know_to_the_general_path():
    fast = binding._fast()
    p, cu, w = torch.zeros((4, 2, 64), dtype=BF), torch.zeros(2, dtype=torch.int32), torch.zeros((3, 2, 16))
    at = (1 << 20, 1, 2, 64, 3, 16)
    assert fast.paged_append(p, p, cu, at, 4, None) is None and fast.paged_append(p, p, cu, None, 4, None) is None and fast.paged_append() is None
    assert fast.paged_forward(p, p, cu, at, 4, 4, True, 0.0, None, None) is None and fast.paged_forward(p, p, cu, at[:5], 4, 4, True, 0.0, None, None) is None
    assert fast.paged_weights(p, w[0], w, cu, at, 4, 4, None, 1.0, True, 0.0) is None
    assert fast.paged_evict(at, w, at, None, torch.zeros((1, 2, 4), dtype=torch.int32), 0, 0) is None and fast.paged_evict(at, w, (1, 2), None, w, 0, 0) is None


def _setting(seed=3):
    dev = "cuda:0"
    g = torch.Generator(device=dev).manual_seed(seed)

    def randn(*shape):
        return torch.randn(shape, generator=g, device=dev).to(BF)

    S, Hq, Hkv, D, page, pages, new = 3, 8, 2, 64, 16, 40, [1, 20, 3]
    cu = torch.tensor([0, 1, 21, 24], dtype=torch.int32, device=dev)
    table = torch.randperm(pages, generator=torch.Generator().manual_seed(1))[:S * 12].view(S, 12).to(torch.int32).to(dev)
    used = torch.tensor([100, 90, 180], dtype=torch.int32, device=dev)
    k, v = randn(pages, page, Hkv, D), randn(pages, page, Hkv, D)
    return randn, S, Hq, Hkv, D, page, pages, cu, table, used, k, v


@pytest.mark.gpu
def test_same_results_both_ways():
    here = torch.cuda.current_stream()
    results = []
    for stream in (None, here):
        randn, S, Hq, Hkv, D, page, pages, cu, table, used, k, v = _setting()
        cache = sta.StaPagedCache(k, v, table, used)
        x, q = randn(24, 2 * Hkv, D), randn(24, Hq, D)
        weights = torch.rand((pages, Hkv, page), generator=torch.Generator(device="cuda:0").manual_seed(5), device="cuda:0")
        assert sta.sta_paged_append(x[:, :Hkv], x[:, Hkv:], cu, cache, 20, weights=weights, stream=stream) is cache
        o, lse = torch.empty_like(q), torch.empty((Hq, 24), device="cuda:0")
        ws = torch.empty(max(16, sta.sta_paged_workspace_bytes(Hq, Hkv, D, S, 24, 20, 192)), dtype=torch.uint8, device="cuda:0")
        assert sta.sta_paged_forward(q, o, cu, cache, 20, 192, lse=lse, workspace=ws, stream=stream) is o
        assert sta.sta_paged_weights(q, lse, weights, cu, cache, 20, 192, before=weights, decay=0.5, stream=stream) is weights
        into = sta.StaPagedCache(torch.zeros_like(k), torch.zeros_like(v), table, torch.zeros_like(used))
        to_w, kept = torch.zeros_like(weights), torch.zeros((S, Hkv, 50), dtype=torch.int32, device="cuda:0")
        assert sta.sta_paged_evict(cache, weights, into, to_w, kept, first=1, recent=8, stream=stream) is into
        results.append([k, v, weights, o, lse, into.k, into.v, into.used, to_w, kept])
    assert all(torch.equal(a, b) for a, b in zip(*results))
    assert results[0][7].tolist() == [50, 50, 50]


@pytest.mark.gpu
def test_same_errors_both_ways():
    randn, S, Hq, Hkv, D, page, pages, cu, table, used, k, v = _setting()
    cache = sta.StaPagedCache(k, v, table, used)
    q, x = randn(24, Hq, D), randn(24, Hkv, D)
    o, lse, w = torch.empty_like(q), torch.empty((Hq, 24), device="cuda:0"), torch.zeros((pages, Hkv, page), device="cuda:0")
    kept = torch.zeros((S, Hkv, 50), dtype=torch.int32, device="cuda:0")
    other = sta.StaPagedCache(k.clone(), v.clone(), table[:2], used[:2])
    for stream in (None, torch.cuda.current_stream()):
        for call, status in ((lambda: sta.sta_paged_forward(q, q, cu, cache, 20, 192, stream=stream), 5), (lambda: sta.sta_paged_forward(q, o, cu, cache, 20, -1, stream=stream), 2),
                             (lambda: sta.sta_paged_append(k[0, :1].expand(24, -1, -1), x, cu, cache, 20, stream=stream), 5),
                             (lambda: sta.sta_paged_weights(q, lse, w, cu, cache, 20, 192, before=w, decay=float("inf"), stream=stream), 4),
                             (lambda: sta.sta_paged_evict(cache, w, cache, w, kept, first=40, recent=11, stream=stream), 2)):
            with pytest.raises(sta.StaError) as e:
                call()
            assert e.value.status == status
        for call, match in ((lambda: sta.sta_paged_forward(q, o, cu[:3], cache, 20, 192, stream=stream), "an entry more"), (lambda: sta.sta_paged_append(x[:, :1], x, cu, cache, 20, stream=stream), "must be"),
                            (lambda: sta.sta_paged_weights(q, lse, w[1:], cu, cache, 20, 192, stream=stream), "weights must be"),
                            (lambda: sta.sta_paged_weights(q, lse, w, cu, cache, 20, 192, before=w[1:], stream=stream), "before must be"),
                            (lambda: sta.sta_paged_weights(q, None, w, cu, cache, 20, 192, stream=stream), "are needed"), (lambda: sta.sta_paged_evict(cache, w, other, None, kept, stream=stream), "same sequences"),
                            (lambda: sta.sta_paged_evict(cache, w, cache, w, kept[:2], stream=stream), "kept must be"), (lambda: sta.sta_paged_evict(cache, None, cache, w, kept, stream=stream), "are needed")):
            with pytest.raises(ValueError, match=match):
                call()
        with pytest.raises(TypeError):
            sta.sta_paged_append(x.half(), x, cu, cache, 20, stream=stream)
