"""The row and packed operators through the extension and through ctypes: the same results, the same errors, and everything that
the extension does not know is left to the general path."""
import pytest
import torch

import paper_2502_04507_amd as sta
from paper_2502_04507_amd import binding

BF = torch.bfloat16


def test_leaves_what_it_does_not_know_to_the_general_path():
    fast = binding._fast()
    x, w, cu = torch.zeros((1, 4, 2, 64), dtype=BF), torch.zeros(64), torch.zeros(2, dtype=torch.int32)
    p = torch.zeros((4, 2, 64), dtype=BF)
    at = (1 << 20, -1, -1)
    assert fast.rope((x,), (x,), at, False) is None and fast.rope(x, x, at, False) is None and fast.rope((), (), at, False) is None
    assert fast.rope((x,), (x,), None, False) is None and fast.rope() is None
    assert fast.norm_rope(x, x, None, x, x, None, w, w, at, 1e-6, None, None) is None
    assert fast.norm_rope_backward(x, x, x, x, None, x, x, None, w, w, w, w, at, w, 1e-6, None, None) is None
    assert fast.packed_forward(p, p, p, p, cu, cu, 4, 4, True, 0.0, None, None, None) is None
    assert fast.packed_backward(p, p, p, p, p, w, p, p, p, cu, cu, 4, 4, w, True, 0.0) is None
    with pytest.raises(ValueError, match="must live in device memory"):
        sta.sta_packed_forward(p, p, p, p, cu, cu, 4, 4)
    with pytest.raises(ValueError, match="must live in device memory"):
        sta.sta_qk_norm_rope(x, x, None, x.clone(), x.clone(), None, w, w, None)
    with pytest.raises(ValueError, match="must be int32"):
        sta.StaRotary(torch.zeros(4, dtype=torch.int64), positions=torch.zeros(3, dtype=torch.int64))


@pytest.mark.gpu
def test_same_results_both_ways():
    dev = "cuda:0"
    g = torch.Generator(device=dev).manual_seed(3)

    def randn(*shape):
        return torch.randn(shape, generator=g, device=dev).to(BF)

    B, N, Hq, Hk, D = 2, 33, 4, 2, 64
    steps, _ = sta.sta_rope_steps(D)
    rotary = sta.StaRotary(steps.to(dev), positions=torch.arange(N, dtype=torch.int32, device=dev) + 5)
    qkv, w = randn(B, N, Hq + 2 * Hk, D), [randn(D), randn(D)]
    q, k, v = qkv.split([Hq, Hk, Hk], 2)
    here = torch.cuda.current_stream()
    results = []
    for stream in (None, here):
        out = [torch.empty((B, h, N, D), dtype=BF, device=dev).transpose(1, 2) for h in (Hq, Hk, Hk)]
        sta.sta_qk_norm_rope(q, k, v, *out, *w, rotary, eps=1e-5, stream=stream)
        d_qkv, dw = torch.empty_like(qkv), [torch.empty(D, device=dev) for _ in range(2)]
        ws = torch.empty(sta.sta_qk_norm_rope_workspace_bytes(D), dtype=torch.uint8, device=dev)
        sta.sta_qk_norm_rope_backward(q, k, *out, *d_qkv.split([Hq, Hk, Hk], 2), *w, *dw, rotary, ws, eps=1e-5, stream=stream)
        turned = [torch.empty_like(x) for x in (q, k)]
        sta.sta_rope((q, k), turned, rotary, inverse=True, stream=stream)
        p = [x.reshape(B * N, -1, D) for x in out]
        cu = torch.tensor([0, 20, B * N], dtype=torch.int32, device=dev)
        o, lse = torch.empty_like(p[0]), torch.empty((Hq, B * N), device=dev)
        sta.sta_packed_forward(*p, o, cu, cu, 46, 46, lse=lse, stream=stream)
        d = [torch.empty_like(x) for x in p]
        ws = torch.empty(sta.sta_packed_backward_workspace_bytes(Hq, B * N), dtype=torch.uint8, device=dev)
        sta.sta_packed_backward(*p, o, p[0], lse, *d, cu, cu, 46, 46, ws, stream=stream)
        results.append(out + [d_qkv, *dw, *turned, o, lse, *d])
    assert all(torch.equal(a, b) for a, b in zip(*results))


@pytest.mark.gpu
def test_same_errors_both_ways():
    dev = "cuda:0"
    steps, _ = sta.sta_rope_steps(64)
    rotary = sta.StaRotary(steps.to(dev), positions=torch.arange(7, dtype=torch.int32, device=dev))
    x = torch.zeros((1, 8, 2, 64), dtype=BF, device=dev)
    p, cu = torch.zeros((8, 2, 64), dtype=BF, device=dev), torch.zeros(2, dtype=torch.int32, device=dev)
    for stream in (None, torch.cuda.current_stream()):
        with pytest.raises(ValueError, match="positions do not match"):
            sta.sta_rope(x, x, rotary, stream=stream)
        with pytest.raises(sta.StaError) as e:              # output in its input
            sta.sta_packed_forward(p, p, p, p, cu, cu, 8, 8, stream=stream)
        assert e.value.status == 5
        with pytest.raises(sta.StaError) as e:              # an output that is its own neighbour
            sta.sta_qk_norm_rope(x, x, None, x[:, :, :1].expand(1, 8, 2, 64), x.clone(), None, None, None, None, stream=stream)
        assert e.value.status == 2
