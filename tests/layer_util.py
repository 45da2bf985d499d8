"""Plain 64-bit implementations of the operators around the attention, on host tensors."""
import math

import numpy as np
import torch


def angles(steps, pairs, positions):
    """[N, pairs] float64: 2 pi frac(x step / 2^64), from whole-number products of any size."""
    axis = [a for a, n in enumerate(pairs) for _ in range(n)]
    out = np.empty((len(positions), len(axis)))
    for i, (s, a) in enumerate(zip(steps, axis)):
        for n, x in enumerate(positions):
            phase = (int(x[a]) * int(s)) % (1 << 64)
            out[n, i] = 2 * math.pi * (phase / 2.0 ** 64)
    return torch.from_numpy(out)


def rotate(x, angle, interleaved, magnitude=1.0, inverse=False):
    """x: [B, N, H, D] float64; angle: [N, pairs] or [B, N, pairs]."""
    pairs = angle.shape[-1]
    angle = angle if angle.dim() == 3 else angle[None]
    c, s = (f(angle)[:, :, None, :] * magnitude for f in (torch.cos, torch.sin))
    if inverse:
        s = -s
    y = x.clone()
    first = slice(0, 2 * pairs, 2) if interleaved else slice(0, pairs)
    second = slice(1, 2 * pairs, 2) if interleaved else slice(pairs, 2 * pairs)
    a, b = x[..., first], x[..., second]
    y[..., first], y[..., second] = a * c - b * s, a * s + b * c
    return y


def norm_rope(x, w, eps, turn):
    """turn: what rotates, a function of rows."""
    r = 1.0 / torch.sqrt((x * x).mean(-1, keepdim=True) + eps)
    return turn(x * r * w)


def norm_rope_backward(x, w, eps, dy, turn_back):
    r = 1.0 / torch.sqrt((x * x).mean(-1, keepdim=True) + eps)
    g = turn_back(dy)
    terms = g * x * r
    gw = g * w
    dx = r * (gw - x * r * r * (gw * x).mean(-1, keepdim=True))
    return dx, terms.sum((0, 1, 2)), terms.abs().sum((0, 1, 2))


def tile_places(grid, tile):
    """Place in tiled order of every raster token."""
    t, h, w = np.meshgrid(*[np.arange(n) for n in grid], indexing="ij")
    x = [a.reshape(-1) for a in (t, h, w)]
    n = [g // s for g, s in zip(grid, tile)]
    tid = ((x[0] // tile[0]) * n[1] + x[1] // tile[1]) * n[2] + x[2] // tile[2]
    inside = ((x[0] % tile[0]) * tile[1] + x[1] % tile[1]) * tile[2] + x[2] % tile[2]
    return torch.from_numpy(tid * (tile[0] * tile[1] * tile[2]) + inside)


def raster_positions(grid):
    return np.stack(np.meshgrid(*[np.arange(n) for n in grid], indexing="ij"), -1).reshape(-1, 3)


def assert_rounded(got, want, slack, label):
    """got equals want but for `slack` (absolute, per element or one number) and one rounding to got's type."""
    unit = 2.0 ** -7 if got.dtype == torch.bfloat16 else 2.0 ** -23        # spacing of numbers in [1, 2): 7 and 23 stored bits
    g = got.detach().cpu().double()
    assert g.shape == want.shape, label
    # a result off by `slack` may round to the neighbour of what the exact one rounds to: half a unit of the larger one
    bound = slack + 0.5 * unit * (want.abs() + slack)
    off = (g - want).abs()
    assert bool((off <= bound).all()), "%s: off by %.3e where %.3e is allowed" % (
        label, float((off - bound).max() + bound.flatten()[(off - bound).argmax()]), float(bound.flatten()[(off - bound).argmax()]))


def seen(lq, lk, causal):
    i = torch.arange(lq)[:, None]
    j = torch.arange(lk)[None, :]
    return (j <= i + lk - lq) if causal else torch.ones((lq, lk), dtype=torch.bool)


def attention(q, k, v, causal, scale, d_o=None):
    """One sequence: q [lq, Hq, D], k and v [lk, Hkv, D] float64.  Keys that a row does not see take no part in it, whatever they hold.
    Returns o, lse [Hq, lq] and with d_o the gradients."""
    lq, Hq, D = q.shape
    lk, Hkv = k.shape[0], k.shape[1]
    keep = seen(lq, lk, causal)
    o = torch.zeros_like(q)
    lse = torch.full((Hq, lq), -math.inf, dtype=torch.float64)
    d = [torch.zeros_like(x) for x in (q, k, v)]
    for h in range(Hq):
        n = h // (Hq // Hkv)
        if lk == 0 or lq == 0:
            continue
        s = torch.where(keep, q[:, h] @ k[:, n].T * scale, -math.inf)
        lse[h] = torch.logsumexp(s, -1)
        p = torch.where(keep, torch.exp(s - torch.where(torch.isinf(lse[h]), 0.0, lse[h])[:, None]), 0.0)
        o[:, h] = p @ v[:, n]
        if d_o is None:
            continue
        g = d_o[:, h]
        ds = p * (g @ v[:, n].T - (g * o[:, h]).sum(-1, keepdim=True)) * scale
        d[0][:, h] = ds @ k[:, n]
        d[1][:, n] += ds.T @ q[:, h]
        d[2][:, n] += p.T @ g
    return (o, lse) if d_o is None else (o, lse, *d)
