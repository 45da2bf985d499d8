"""Norms and rotary positions of query and key rows on the GPU, against the formulas in 64 bits.

Allowed errors.  Inputs are the same numbers on both sides.  In fp32 the norm's factor is a sum of D squares by 16 products a lane and
a few exchanges, a reciprocal root and two products: below 16 units of 2^-24 relative.  Cosines and sines are within 2^-23; a rotated
channel is two products and a sum: 4 units of 2^-24 of |a| + |b| more.  So 32 units of 2^-24 of the row's largest channel times sqrt 2
and the magnitude bound it, and one rounding to the output's type comes on top.  Gradients pass through the same steps twice and
a second sum over the row: 96 units.  Weight gradients are sums of terms with that error, added a few hundred at a time in a row:
512 units of the terms' absolute sum."""
import numpy as np
import pytest
import torch

import paper_2502_04507_amd as sta
from tests import layer_util as lu

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
ULP = 2.0 ** -24


def make(shape, seed, dtype, spread=1.0):
    g = torch.Generator().manual_seed(seed)
    return (torch.randn(shape, generator=g) * spread).to(dtype)


def rotary_of(rot, pairs, interleaved, N, start=0, magnitude=1.0, grid=None, explicit=True, batches=None):
    steps = torch.cat([sta.sta_rope_steps(2 * n)[0] for n in pairs if n])
    if grid is not None:
        positions = lu.raster_positions(grid)
    else:
        positions = np.arange(start, start + N)[:, None]
    dev = None
    if explicit:
        p = torch.from_numpy(positions.astype(np.int32))
        dev = (p if len(pairs) == 3 else p[:, 0]).contiguous().to(DEV)
    return (sta.StaRotary(steps.to(DEV), positions=dev, pairs=pairs, interleaved=interleaved, magnitude=magnitude),
            lu.angles(steps.tolist(), pairs, positions))


def slack(x, units, magnitude=1.0):
    return units * ULP * 1.5 * magnitude * x.abs().amax(-1, keepdim=True).expand_as(x) + 1e-30


# B, N, heads, D, rot, interleaved
ROPE = [
    (1, 1, (1,), 64, 64, False), (2, 9, (3, 1), 64, 64, True), (1, 17, (4, 2), 128, 128, False), (3, 5, (5, 1, 2), 128, 64, True),
    (1, 33, (2, 2), 128, 32, False), (2, 7, (3, 3), 80, 80, False), (2, 7, (3,), 80, 40, True), (1, 11, (2, 1), 80, 40, False),
    (1, 5, (2,), 80, 20, True), (1, 9, (2, 2), 96, 48, False), (1, 6, (3,), 96, 24, False), (1, 13, (2, 1), 256, 256, True),
    (1, 3, (1, 1), 256, 128, False), (1, 3, (2,), 2, 2, True), (1, 4, (3,), 6, 4, False), (2, 300, (1,), 16, 16, True),
    (1, 5, (33, 9), 48, 32, False), (1, 5, (3,), 130, 66, False),
    # aligned rows whose pairs or chunks are split by lanes
    (2, 19, (3, 2), 64, 8, False), (1, 21, (2,), 256, 40, False), (1, 7, (5,), 128, 2, True), (1, 9, (4, 1), 96, 94, False), (3, 4, (2, 2), 128, 100, True),
    (1, 40, (1,), 16, 6, False),
]


def many(B, N, heads, D):
    """Batch entries that make more than 2^21 channels: launches of fewer may go to another kernel."""
    return max(B, 2 ** 21 // (N * heads * D) + 1)


@pytest.mark.parametrize("src,dst", [("bf16", "bf16"), ("f32", "f32"), ("f32", "bf16"), ("bf16", "f32")])
@pytest.mark.parametrize("B,N,heads,D,rot,interleaved", ROPE)
def test_rope(B, N, heads, D, rot, interleaved, src, dst):
    check_rope(B, N, heads, D, rot, interleaved, src, dst)


@pytest.mark.parametrize("src,dst", [("bf16", "bf16"), ("f32", "f32"), ("f32", "bf16"), ("bf16", "f32")])
@pytest.mark.parametrize("B,N,heads,D,rot,interleaved", [c for c in ROPE if c[3] % 16 == 0 and c[4] % 8 == 0])
def test_rope_of_many_rows(B, N, heads, D, rot, interleaved, src, dst):
    check_rope(many(B, N, sum(heads), D), N, heads, D, rot, interleaved, src, dst)


def check_rope(B, N, heads, D, rot, interleaved, src, dst):
    types = {"bf16": torch.bfloat16, "f32": torch.float32}
    xs = [make((B, N, h, D), 5 + i, types[src]) for i, h in enumerate(heads)]
    rotary, angle = rotary_of(rot, (rot // 2,), interleaved, N, start=1000003, magnitude=1.25)
    for inverse in (False, True):
        outs = [torch.full(x.shape, float("nan"), dtype=types[dst], device=DEV) for x in xs]
        sta.sta_rope([x.to(DEV) for x in xs], outs, rotary, inverse=inverse)
        for x, y in zip(xs, outs):
            want = lu.rotate(x.double(), angle, interleaved, 1.25, inverse)
            lu.assert_rounded(y, want, slack(x.double(), 32, 1.25), "rope inverse=%s" % inverse)
            assert torch.equal(y[..., rot:].cpu().double(), x[..., rot:].to(types[dst]).double())      # the rest is copied


@pytest.mark.parametrize("batches", [1, 1040])
@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("start", [0, 2 ** 20 + 1, 2 ** 31 - 8, -(2 ** 31), -3])
def test_rope_far_positions(start, interleaved, batches):
    x = make((batches, 8, 2, 128), 3, torch.float32)
    rotary, angle = rotary_of(128, (64,), interleaved, 8, start=start)
    y = torch.empty(x.shape, device=DEV)
    sta.sta_rope(x.to(DEV), y, rotary)
    lu.assert_rounded(y, lu.rotate(x.double(), angle, interleaved), slack(x.double(), 32), "rope at %d" % start)


@pytest.mark.parametrize("N", [19, 1500])
def test_rope_in_place_inside_a_fused_tensor_and_per_batch_positions(N):
    B, D = 2, 128
    qkv = make((B, N, 8, D), 7, torch.bfloat16)
    steps = sta.sta_rope_steps(D)[0]
    positions = torch.randint(0, 50000, (B, N), generator=torch.Generator().manual_seed(1), dtype=torch.int32)
    rotary = sta.StaRotary(steps.to(DEV), positions=positions.to(DEV))
    dev = qkv.to(DEV)
    q, k = dev[:, :, :4], dev[:, :, 4:6]
    sta.sta_rope((q, k), (q, k), rotary)
    angle = torch.stack([lu.angles(steps.tolist(), (D // 2,), p.numpy()[:, None]) for p in positions])
    want = lu.rotate(qkv[:, :, :6].double(), angle, False)
    lu.assert_rounded(dev[:, :, :6], want, slack(qkv[:, :, :6].double(), 32), "in place")
    assert torch.equal(dev[:, :, 6:].cpu(), qkv[:, :, 6:])


@pytest.mark.parametrize("D,offset,pad", [(128, 1, 0), (64, 0, 3), (128, 8, 8), (64, 4, 4)])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("N", [21, 5600])
def test_rows_at_any_address_and_stride(N, D, offset, pad, dtype):
    """Rows that start at single elements, wider apart than they are long."""
    B, H = 2, 3
    flat = make((offset + B * N * H * (D + pad) + 64,), 11, dtype)
    view = (B, N, H, D), (N * H * (D + pad), D + pad, N * (D + pad), 1)       # head-major inside a batch
    x = flat.as_strided(*view, offset)
    dev = flat.to(DEV)
    out = torch.full_like(dev, 7.0)
    rotary, angle = rotary_of(D, (D // 2,), True, N)
    sta.sta_rope(dev.as_strided(*view, offset), out.as_strided(*view, offset), rotary)
    lu.assert_rounded(out.as_strided(*view, offset), lu.rotate(x.double(), angle, True), slack(x.double(), 32), "strided")
    written = torch.zeros(flat.shape, dtype=torch.bool)
    written.as_strided(*view, offset).fill_(True)
    assert bool((out.cpu()[~written] == 7.0).all())


def test_rope_of_broadcast_rows():
    x = make((1, 5, 1, 64), 13, torch.bfloat16)
    rotary, angle = rotary_of(64, (32,), False, 5)
    y = torch.empty((3, 5, 4, 64), dtype=torch.bfloat16, device=DEV)
    sta.sta_rope(x.to(DEV).expand(3, 5, 4, 64), y, rotary)
    x = x.expand(3, 5, 4, 64).double()
    lu.assert_rounded(y, lu.rotate(x, angle, False), slack(x, 32), "broadcast")


# B, grid or N, tile, Hq, Hkv, D, rot, interleaved, values
NORM = [
    (1, 1, None, 4, 1, 128, 128, False, True), (4, 3, None, 3, 3, 64, 64, True, False), (1, 130, None, 8, 2, 128, 64, False, True),
    (2, 31, None, 5, 1, 80, 80, False, True), (1, 9, None, 2, 2, 80, 20, True, True), (1, 7, None, 3, 1, 256, 256, False, True),
    (1, 5, None, 2, 1, 10, 6, False, True), (1, (4, 8, 8), (2, 4, 8), 3, 3, 64, 64, True, True),
    (2, (3, 10, 14), (3, 5, 7), 2, 2, 128, 128, True, True), (1, (1, 16, 24), (1, 8, 8), 5, 5, 64, 64, False, True),
    (1, (6, 8, 8), None, 2, 2, 128, 96, True, True), (1, (12, 24, 24), (6, 8, 8), 1, 1, 128, 128, True, True), (3, 700, None, 1, 1, 64, 0, False, True),
    (2, 45, None, 3, 2, 96, 24, False, True), (1, 77, None, 2, 1, 256, 200, False, True), (1, (4, 8, 8), (2, 4, 8), 2, 2, 80, 20, True, True),
]


@pytest.mark.parametrize("src,dst", [("bf16", "bf16"), ("f32", "bf16"), ("f32", "f32"), ("bf16", "f32")])
@pytest.mark.parametrize("case", NORM, ids=[str(i) for i in range(len(NORM))])
def test_norm_rope_and_gradients(case, src, dst):
    check_norm_rope(case, src, dst)


@pytest.mark.parametrize("src,dst", [("bf16", "bf16"), ("f32", "bf16"), ("f32", "f32"), ("bf16", "f32")])
@pytest.mark.parametrize("case", [c for c in NORM if c[5] % 16 == 0 and c[6] % 8 == 0], ids=lambda c: "-".join(str(x) for x in c).replace(" ", ""))
def test_norm_rope_and_gradients_of_many_rows(case, src, dst):
    B, where, tile, Hq, Hkv, D = case[:6]
    N = where[0] * where[1] * where[2] if isinstance(where, tuple) else where
    check_norm_rope((many(B, N, Hq + Hkv, D),) + case[1:], src, dst)


def check_norm_rope(case, src, dst):
    B, where, tile, Hq, Hkv, D, rot, interleaved, values = case
    types = {"bf16": torch.bfloat16, "f32": torch.float32}
    grid = where if isinstance(where, tuple) else None
    N = grid[0] * grid[1] * grid[2] if grid else where
    heads = [Hq, Hkv] + ([Hkv] if values else [])
    eps = 1e-5
    qkv = make((B, N, Hq + 2 * Hkv, D), 21, types[src], 3.0)
    qkv[:, N // 2] *= 1e-4                                  # a token whose mean square is near eps
    ins = list(qkv.split([Hq, Hkv, Hkv], 2))[:len(heads)]
    w = [make((D,), 31 + i, types[dst], 0.5) + 1.0 for i in range(2)]
    rotary, angle = None, None
    if rot:
        side = rot * 7 // 32
        pairs = (rot // 2 - 2 * side, side, side) if grid else (rot // 2,)
        rotary, angle = rotary_of(rot, pairs, interleaved, N, grid=grid, explicit=False)

    def turn(x, inverse=False):
        return x if angle is None else lu.rotate(x, angle, interleaved, 1.0, inverse)

    place = lu.tile_places(grid, tile) if tile else torch.arange(N)
    order = torch.argsort(place)
    dev = list(qkv.to(DEV).split([Hq, Hkv, Hkv], 2))[:len(heads)]
    outs = [torch.full((B, h, N, D), float("nan"), dtype=types[dst], device=DEV).transpose(1, 2) for h in heads]
    v, v_out = (dev[2], outs[2]) if values else (None, None)
    wd = [x.to(DEV) for x in w]
    sta.sta_qk_norm_rope(dev[0], dev[1], v, outs[0], outs[1], v_out, *wd, rotary, eps=eps, grid=grid, tile=tile)
    for i, (x, y) in enumerate(zip(ins, outs)):
        want = lu.norm_rope(x.double(), w[i].double(), eps, turn) if i < 2 else x.double()
        lu.assert_rounded(y, want[:, order], slack(want, 32)[:, order] if i < 2 else torch.zeros_like(want), "output %d" % i)

    dy = [make((B, h, N, D), 41 + i, types[dst]).transpose(1, 2) for i, h in enumerate(heads)]
    dyd = [x.to(DEV) for x in dy]
    d_qkv = torch.full(qkv.shape, float("nan"), dtype=types[src], device=DEV)
    dx = list(d_qkv.split([Hq, Hkv, Hkv], 2))[:len(heads)]
    dw = [torch.full((D,), float("nan"), device=DEV) for _ in range(2)]
    ws = torch.full((sta.sta_qk_norm_rope_workspace_bytes(D),), 255, dtype=torch.uint8, device=DEV)
    again = None
    for _ in range(2):
        sta.sta_qk_norm_rope_backward(dev[0], dev[1], dyd[0], dyd[1], dyd[2] if values else None, dx[0], dx[1], dx[2] if values else None,
                                      *wd, *dw, rotary, ws, eps=eps, grid=grid, tile=tile)
        now = [t.clone() for t in dx + dw]
        assert again is None or all(torch.equal(a, b) for a, b in zip(again, now))
        again = now
    for i, g in enumerate(dy):
        g = g.double()[:, place]
        if i == 2:
            lu.assert_rounded(dx[2], g, torch.zeros_like(g), "d_v")
            continue
        x, weight = ins[i].double(), w[i].double()
        want, sums, absolute = lu.norm_rope_backward(x, weight, eps, g, lambda t: turn(t, True))
        r = 1.0 / torch.sqrt((x * x).mean(-1, keepdim=True) + eps)
        size = r * (g.abs().amax(-1, keepdim=True) * weight.abs().max() * 1.5) * (1 + (x * r).abs().amax(-1, keepdim=True) ** 2)
        lu.assert_rounded(dx[i], want, (96 * ULP * size).expand_as(want), "gradient %d" % i)
        lu.assert_rounded(dw[i], sums, 512 * ULP * absolute + 1e-30, "weight gradient %d" % i)


def test_gradients_against_differences():
    """The loss sum(y o g) moves by h times the gradient along random directions; central differences in 64 bits of the formula."""
    B, N, H, D, eps = 1, 6, 2, 64, 1e-6
    x, g, w = make((B, N, H, D), 51, torch.float32), make((B, N, H, D), 52, torch.float32), make((D,), 53, torch.float32) + 1.0
    rotary, angle = rotary_of(D, (D // 2,), False, N, start=77)
    dev = [t.to(DEV) for t in (x, g, w)]
    dx, dw = [torch.empty_like(dev[0]) for _ in range(2)], [torch.empty(D, device=DEV) for _ in range(2)]
    ws = torch.empty(sta.sta_qk_norm_rope_workspace_bytes(D), dtype=torch.uint8, device=DEV)
    sta.sta_qk_norm_rope_backward(dev[0], dev[0], dev[1], dev[1], None, dx[0], dx[1], None, dev[2], dev[2], *dw, rotary, ws, eps=eps)

    def loss(x, w):
        return float((lu.norm_rope(x, w, eps, lambda t: lu.rotate(t, angle, False)) * g.double()).sum())

    for seed in range(4):
        u, uw = make(x.shape, 60 + seed, torch.float64), make(w.shape, 70 + seed, torch.float64)
        h = 1e-5
        want = (loss(x.double() + h * u, w.double() + h * uw) - loss(x.double() - h * u, w.double() - h * uw)) / (2 * h)
        parts = (dx[0].cpu().double() * u).abs().sum() + (dw[0].cpu().double() * uw).abs().sum()
        got = float((dx[0].cpu().double() * u).sum() + (dw[0].cpu().double() * uw).sum())
        assert abs(got - want) <= 1e-5 * float(parts), (got, want)


def test_weight_gradients_of_no_tokens_are_zero():
    q = torch.empty((2, 0, 3, 64), dtype=torch.bfloat16, device=DEV)
    dw = [torch.full((64,), float("nan"), device=DEV) for _ in range(2)]
    ws = torch.empty(sta.sta_qk_norm_rope_workspace_bytes(64), dtype=torch.uint8, device=DEV)
    sta.sta_qk_norm_rope(q, q, None, q.clone(), q.clone(), None, None, None, None)
    sta.sta_qk_norm_rope_backward(q, q, q, q, None, q.clone(), q.clone(), None, None, None, *dw, None, ws)
    assert all(bool((x == 0).all()) for x in dw)


@pytest.mark.parametrize("N", [300, 5000])
def test_another_stream_and_a_graph(N):
    x = make((1, N, 4, 128), 81, torch.bfloat16).to(DEV)
    rotary, angle = rotary_of(128, (64,), False, N)
    want = torch.empty_like(x)
    sta.sta_rope(x, want, rotary)
    y = torch.empty_like(x)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    sta.sta_rope(x, y, rotary, stream=s)
    s.synchronize()
    assert torch.equal(y, want)
    graph = torch.cuda.CUDAGraph()
    w = torch.ones(128, device=DEV)
    q = torch.empty_like(x)
    with torch.cuda.graph(graph):
        sta.sta_qk_norm_rope(x, x, None, y, q, None, w, w, rotary)
    for seed in (1, 2, 3):
        x.copy_(make(x.shape, seed, torch.bfloat16))
        graph.replay()
        a, b = torch.empty_like(x), torch.empty_like(x)
        sta.sta_qk_norm_rope(x, x, None, a, b, None, w, w, rotary)
        torch.cuda.synchronize()
        assert torch.equal(a, y) and torch.equal(b, q)


def test_rows_beyond_4_gb():
    """The last tokens of a tensor whose offsets pass 32 bits, forward and backward, against the same rows alone."""
    N, D, n = 9_000_000, 256, 9000
    x = torch.zeros((1, N, 1, D), dtype=torch.bfloat16, device=DEV)
    assert x.numel() * 2 > 2 ** 32
    tail = make((1, n, 1, D), 3, torch.bfloat16).to(DEV)
    x[:, -n:] = tail
    steps = sta.sta_rope_steps(D)[0].to(DEV)
    w = torch.ones(D, device=DEV)
    positions = torch.arange(N, dtype=torch.int32, device=DEV)
    big, small = sta.StaRotary(steps), sta.StaRotary(steps, positions=positions[-n:].clone())
    y, z = torch.empty_like(x), torch.empty_like(tail)
    sta.sta_rope(x, y, big)
    sta.sta_rope(tail, z, small)
    assert torch.equal(y[:, -n:], z)
    k, k_out = x[:, :, :, :].narrow(1, 0, N), torch.empty_like(x)
    sta.sta_qk_norm_rope(x, k, None, y, k_out, None, w, None, big)
    sta.sta_qk_norm_rope(tail, tail, None, z, torch.empty_like(tail), None, w, None, small)
    assert torch.equal(y[:, -n:], z) and torch.equal(k_out[:, -n:], z)
    d, dz = [k_out, torch.empty_like(x)], [torch.empty_like(tail) for _ in range(2)]
    sta.sta_qk_norm_rope_backward(x, x, y, y, None, *d, None, w, None, None, None, big, None)
    sta.sta_qk_norm_rope_backward(tail, tail, z, z, None, *dz, None, w, None, None, None, small, None)
    assert torch.equal(d[0][:, -n:], dz[0]) and torch.equal(d[1][:, -n:], dz[1])


def test_rows_of_more_than_2_to_the_24_workgroups():
    """Tokens beyond 2^24 of rows that take a wave each: those around the places where the grid is folded, and the last, against the same rows alone."""
    N, D, n = 2 ** 24 + 777, 130, 300
    x = torch.zeros((1, N, 1, D), dtype=torch.bfloat16, device=DEV)
    steps = sta.sta_rope_steps(D)[0].to(DEV)
    w = torch.ones(D, device=DEV)
    places = [slice(a, a + n) for a in (0, 2 ** 23 - 150, 2 ** 24 - 150, N - n)]
    for i, at in enumerate(places):
        x[:, at] = make((1, n, 1, D), 3 + i, torch.bfloat16).to(DEV)
    turned, normed, other = torch.empty_like(x), torch.empty_like(x), torch.empty_like(x)
    sta.sta_rope(x, turned, sta.StaRotary(steps))
    sta.sta_qk_norm_rope(x, x, None, normed, other, None, w, None, sta.StaRotary(steps))
    for at in places:
        positions = torch.arange(at.start, at.stop, dtype=torch.int32, device=DEV)
        rotary, rows = sta.StaRotary(steps, positions=positions), x[:, at].contiguous()
        a, b, c = (torch.empty_like(rows) for _ in range(3))
        sta.sta_rope(rows, a, rotary)
        sta.sta_qk_norm_rope(rows, rows, None, b, c, None, w, None, rotary)
        assert torch.equal(turned[:, at], a) and torch.equal(normed[:, at], b) and torch.equal(other[:, at], c), at


@pytest.mark.parametrize("N", [33, 900])
@pytest.mark.parametrize("layout", ["head-major", "cache", "token-major"])
def test_outputs_side_by_side_in_one_tensor(layout, N):
    """Queries, keys and values of two batch entries as views of one allocation, whose spans meet though no element does."""
    B, Hq, Hkv, D = 2, 4, 2, 64
    heads, slots = [Hq, Hkv, Hkv], N + 7
    qkv, w = make((B, N, sum(heads), D), 3, torch.bfloat16).to(DEV), [make((D,), 4 + i, torch.float32).to(DEV) for i in range(2)]
    ins = qkv.split(heads, 2)
    rotary, _ = rotary_of(D, (D // 2,), False, N)
    want = [torch.empty((B, N, h, D), dtype=torch.bfloat16, device=DEV) for h in heads]
    sta.sta_qk_norm_rope(*ins, *want, *w, rotary)
    if layout == "head-major":
        room = torch.full((B, sum(heads), N, D), 7.0, dtype=torch.bfloat16, device=DEV)
        outs = room.transpose(1, 2).split(heads, 2)
    elif layout == "cache":
        room = torch.full((B, 2, Hkv, slots, D), 7.0, dtype=torch.bfloat16, device=DEV)
        outs = [torch.empty_like(want[0])] + [room[:, i, :, :N].transpose(1, 2) for i in range(2)]
    else:
        room = torch.full((B, N * sum(heads) * D + 8), 7.0, dtype=torch.bfloat16, device=DEV)
        outs = room[:, :-8].unflatten(1, (N, sum(heads), D)).split(heads, 2)
    sta.sta_qk_norm_rope(*ins, *outs, *w, rotary)
    assert all(torch.equal(a, b) for a, b in zip(outs, want))
    if layout == "cache":
        assert bool((room[:, :, :, N:] == 7.0).all())
    if layout == "token-major":
        assert bool((room[:, -8:] == 7.0).all())
    turned = [torch.empty_like(x) for x in want[:2]]
    sta.sta_rope(want[:2], turned, rotary)
    sta.sta_rope(outs[:2], outs[:2], rotary)                # in place, next to each other
    assert all(torch.equal(a, b) for a, b in zip(outs[:2], turned)) and torch.equal(outs[2], want[2])
    grads = [make((B, N, h, D), 9 + i, torch.bfloat16).to(DEV) for i, h in enumerate(heads)]
    d_want = [torch.empty_like(x) for x in want]
    d_outs = torch.empty((B, sum(heads), N, D), dtype=torch.bfloat16, device=DEV).transpose(1, 2).split(heads, 2)
    for d in (d_want, d_outs):
        sta.sta_qk_norm_rope_backward(ins[0], ins[1], *grads, *d, *w, None, None, rotary, None)
    assert all(torch.equal(a, b) for a, b in zip(d_outs, d_want))


@pytest.mark.parametrize("N", [9, 6003])
@pytest.mark.parametrize("heads", [3, 8])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_weight_gradients_of_an_infinity(N, heads, dtype):
    """An infinite gradient of the first token's, or the last head's, row makes an infinite weight gradient: rows that are not there add nothing."""
    D, eps = 128, 1e-5
    x, w = make((1, N, heads, D), 3, dtype), make((D,), 4, torch.float32) + 1.0
    dy = [make((1, N, heads, D), 5 + i, dtype) for i in range(2)]
    dy[0][0, 0, 0, 7], dy[1][0, N // 2, heads - 1, 30] = float("inf"), -float("inf")
    dw = [torch.empty(D, device=DEV) for _ in range(2)]
    dx = [torch.empty_like(x, device=DEV) for _ in range(2)]
    ws = torch.empty(sta.sta_qk_norm_rope_workspace_bytes(D), dtype=torch.uint8, device=DEV)
    xd, wd = x.to(DEV), w.to(DEV)
    sta.sta_qk_norm_rope_backward(xd, xd, dy[0].to(DEV), dy[1].to(DEV), None, *dx, None, wd, wd, *dw, None, ws, eps=eps)
    for got, g, at in ((dw[0], dy[0], (0, 0, 0, 7)), (dw[1], dy[1], (0, N // 2, heads - 1, 30))):
        assert float(got[at[-1]]) == float(g[at]) * float(torch.sign(x[at]))
        g = g.clone()
        g[at] = 0.0
        _, sums, absolute = lu.norm_rope_backward(x.double(), w.double(), eps, g.double(), lambda t: t)
        others = torch.arange(D) != at[-1]
        lu.assert_rounded(got.cpu()[others], sums[others], (512 * ULP * absolute + 1e-30)[others], "weight gradient")
