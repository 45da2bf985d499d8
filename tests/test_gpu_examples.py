"""The example layers run, and agree with the formulas on small sizes."""
import importlib.util
import os

import pytest
import torch

import paper_2502_04507_amd as sta
from tests import layer_util as lu

pytestmark = pytest.mark.gpu
ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def example():
    spec = importlib.util.spec_from_file_location("transformer_layers", os.path.join(ROOT, "examples", "transformer_layers.py"))
    module = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(module)
    return module


def test_layers_run_and_next_tokens_continue_prompts():
    # both round probabilities and results to bf16: each is within 2^-7 of the rows' size, see the packed attention's tests
    assert example().main() < 1e-2


def test_prompt_layer_and_its_gradients_against_64_bits():
    """The whole layer: norms, rotation, causal attention, and back.  Rounded to bf16 four times on the way forward and five on the way back, every
    time with a relative error of at most 2^-8 of what is rounded: 2-norms within 2e-2 and 4e-2."""
    ex = example()
    Hq, Hkv, D, lengths = 4, 2, 64, [40, 9]
    T = sum(lengths)
    g = torch.Generator().manual_seed(5)
    qkv, d_o = (torch.randn(s, generator=g).to(torch.bfloat16) for s in ((1, T, Hq + 2 * Hkv, D), (T, Hq, D)))
    w = [1.0 + 0.2 * torch.randn(D, generator=g) for _ in range(2)]
    o, _, _, d_qkv, d_w = ex.prompt_layer(qkv.cuda(), d_o.cuda(), [x.cuda() for x in w], lengths, Hq, Hkv)
    steps, magnitude = sta.sta_rope_steps(D, theta=500000.0, scaling=sta.STA_ROPE_YARN, factor=4.0, original_positions=8192)
    positions = torch.cat([torch.arange(n) for n in lengths]).numpy()[:, None]
    angle = lu.angles(steps.tolist(), (D // 2,), positions)
    x = qkv.double().requires_grad_()
    w64 = [t.double().requires_grad_() for t in w]
    q, k, v = x.split([Hq, Hkv, Hkv], 2)

    def rotated(t):
        c, s = torch.cos(angle)[None, :, None] * magnitude, torch.sin(angle)[None, :, None] * magnitude
        a, b = t[..., :D // 2], t[..., D // 2:]
        return torch.cat((a * c - b * s, a * s + b * c), -1)

    q, k = (rotated(t / torch.sqrt((t * t).mean(-1, keepdim=True) + 1e-6) * ww)[0] for t, ww in ((q, w64[0]), (k, w64[1])))
    outs, at = [], 0
    for n in lengths:
        rows = slice(at, at + n)
        at += n
        keys, values = (t[rows].repeat_interleave(Hq // Hkv, 1).transpose(0, 1) for t in (k, v[0]))
        s = (q[rows].transpose(0, 1) @ keys.transpose(1, 2)) * D ** -0.5
        s = s.masked_fill(~torch.ones(n, n, dtype=torch.bool).tril(), float("-inf"))
        outs.append((torch.softmax(s, -1) @ values).transpose(0, 1))
    want = torch.cat(outs)
    want.backward(d_o.double())

    def rel(a, b):
        return float((a.cpu().double() - b).norm() / b.norm())

    assert rel(o, want.detach()) < 2e-2
    assert rel(d_qkv, x.grad) < 4e-2 and rel(d_w[0], w64[0].grad) < 4e-2 and rel(d_w[1], w64[1].grad) < 4e-2


def test_video_layer_is_its_parts():
    """The fused pass into tile order gives what the norm, the rotation and the permutation give one after the other, but for their rounding between."""
    ex = example()
    grid, tile, H, D = (2, 16, 24), (2, 8, 8), 2, 64
    N = 2 * 16 * 24
    g = torch.Generator().manual_seed(6)
    qkv, d_o = (torch.randn(s, generator=g).to(torch.bfloat16).cuda() for s in ((1, N, 3 * H, D), (1, H, N, D)))
    w = [torch.ones(D).cuda() for _ in range(2)]
    windows = [(1, 3, 3)] * H
    o, d_qkv, d_w = ex.video_layer(qkv, d_o, w, grid, tile, windows)
    side = 7 * D // 32
    pairs = (D // 2 - 2 * side, side, side)
    steps = torch.cat([sta.sta_rope_steps(2 * n, theta=256.0)[0] for n in pairs])
    angle = lu.angles(steps.tolist(), pairs, lu.raster_positions(grid))
    parts = []
    for x in qkv.cpu().split(H, 2)[:2]:
        y = lu.norm_rope(x.double(), torch.ones(D, dtype=torch.float64), 1e-6, lambda t: lu.rotate(t, angle, True))
        parts.append(y.to(torch.bfloat16).transpose(1, 2).contiguous().cuda())
    parts.append(qkv.split(H, 2)[2].transpose(1, 2).contiguous())
    tiled = [sta.sta_tile_permute(p, torch.empty_like(p), grid, tile) for p in parts]
    o_tiled = sta.sta_forward(*tiled, torch.empty_like(tiled[0]), grid, tile, windows)
    want = sta.sta_untile(o_tiled, torch.empty_like(o_tiled), grid, tile)
    assert float((o.float() - want.float()).norm() / want.float().norm()) < 2e-3        # q and k may round to the other neighbour here and there
    assert bool(torch.isfinite(d_qkv.float()).all()) and all(bool(torch.isfinite(x).all()) for x in d_w)
