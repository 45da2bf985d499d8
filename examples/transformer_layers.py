"""Two attention layers of a model that makes video from text, on random weights: what stands between a layer's fused projection and its
attention, and the attention itself, forward, backward and token by token.

  python examples/transformer_layers.py

video_layer    projection -> norms, rotation by (t, h, w) and tile order in one pass -> sliding tile attention -> raster order, and
               the gradients back to the projection's output and the norms' weights;
prompt_layer   the same for packed prompts of different lengths with grouped heads -> causal attention, and its gradients;
next_tokens    one further token of every prompt against a cache of keys and values;
conversation   prompts, the part of them that is looked at, and next tokens with a cache in pages, which is cut to a budget of keys.
"""
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
import paper_2502_04507_amd as sta  # noqa: E402

DEVICE = "cuda:0"
BF16 = torch.bfloat16


def scratch(nbytes):
    return torch.empty(max(16, nbytes), dtype=torch.uint8, device=DEVICE)


def video_layer(qkv, d_o, weights, grid, tile, windows):
    """qkv: [1, N, 3 H, D] as the projection leaves it, tokens in raster order; d_o: gradient of the output, [1, H, N, D] in raster order.
    Returns the output [1, H, N, D], the gradients of qkv and of the norms' weights."""
    B, N, H3, D = qkv.shape
    H = H3 // 3
    # an eighth of the channels turns with time, the rest in equal parts with height and width
    side = 7 * D // 32
    pairs = (D // 2 - 2 * side, side, side)
    steps = torch.cat([sta.sta_rope_steps(2 * n, theta=256.0)[0] for n in pairs]).to(DEVICE)
    rotary = sta.StaRotary(steps, pairs=pairs, interleaved=True)        # positions: the places in the grid
    q, k, v = qkv.split(H, 2)
    tiled = [torch.empty((B, H, N, D), dtype=BF16, device=DEVICE) for _ in range(3)]
    rows = [t.transpose(1, 2) for t in tiled]                           # the same memory as [B, N, H, D]
    sta.sta_qk_norm_rope(q, k, v, *rows, *weights, rotary, grid=grid, tile=tile)
    o_tiled, lse = torch.empty_like(tiled[0]), torch.empty((B, H, N), device=DEVICE)
    sta.sta_forward_lse(*tiled, o_tiled, lse, grid, tile, windows)
    o = sta.sta_untile(o_tiled, torch.empty_like(o_tiled), grid, tile)

    d_o_tiled = sta.sta_tile_permute(d_o, torch.empty_like(d_o), grid, tile)
    d_tiled = [torch.empty_like(t) for t in tiled]
    sta.sta_backward(*tiled, o_tiled, d_o_tiled, lse, *d_tiled, grid, tile, windows, scratch(sta.sta_backward_workspace_bytes(B, H, grid)))
    d_qkv, d_weights = torch.empty_like(qkv), [torch.empty(D, device=DEVICE) for _ in range(2)]
    sta.sta_qk_norm_rope_backward(q, k, *[t.transpose(1, 2) for t in d_tiled], *d_qkv.split(H, 2), *weights, *d_weights, rotary,
                                  scratch(sta.sta_qk_norm_rope_workspace_bytes(D)), grid=grid, tile=tile)
    return o, d_qkv, d_weights


def prompt_rotary(D, positions):
    steps, magnitude = sta.sta_rope_steps(D, theta=500000.0, scaling=sta.STA_ROPE_YARN, factor=4.0, original_positions=8192)
    return sta.StaRotary(steps.to(DEVICE), positions=positions, magnitude=magnitude)


def starts(lengths):
    return torch.tensor([sum(lengths[:i]) for i in range(len(lengths) + 1)], dtype=torch.int32, device=DEVICE)


def prompt_layer(qkv, d_o, weights, lengths, Hq, Hkv):
    """qkv: [1, tokens, Hq + 2 Hkv, D], prompt after prompt; d_o: [tokens, Hq, D].  Returns o, the normed and rotated keys and the values, and the
    gradients of qkv and of the norms' weights."""
    _, T, _, D = qkv.shape
    heads = [Hq, Hkv, Hkv]
    positions = torch.cat([torch.arange(n, dtype=torch.int32) for n in lengths]).to(DEVICE)
    rotary = prompt_rotary(D, positions)
    ins = qkv.split(heads, 2)
    rows = [torch.empty((1, T, h, D), dtype=BF16, device=DEVICE) for h in heads]
    sta.sta_qk_norm_rope(*ins, *rows, *weights, rotary)
    q, k, v = (r[0] for r in rows)
    cu, longest = starts(lengths), max(lengths)
    o, lse = torch.empty_like(q), torch.empty((Hq, T), device=DEVICE)
    sta.sta_packed_forward(q, k, v, o, cu, cu, longest, longest, lse=lse)

    d_rows = [torch.empty_like(r) for r in rows]
    sta.sta_packed_backward(q, k, v, o, d_o, lse, *[r[0] for r in d_rows], cu, cu, longest, longest, scratch(sta.sta_packed_backward_workspace_bytes(Hq, T)))
    d_qkv, d_weights = torch.empty_like(qkv), [torch.empty(D, device=DEVICE) for _ in range(2)]
    sta.sta_qk_norm_rope_backward(ins[0], ins[1], *d_rows, *d_qkv.split(heads, 2), *weights, *d_weights, rotary,
                                  scratch(sta.sta_qk_norm_rope_workspace_bytes(D)))
    return o, k, v, d_qkv, d_weights


class Cache:
    """Keys and values of S sequences, `slot` tokens each."""

    def __init__(self, S, slot, Hkv, D):
        self.k, self.v = (torch.zeros((S * slot, Hkv, D), dtype=BF16, device=DEVICE) for _ in range(2))
        self.first = torch.arange(S + 1, dtype=torch.int32, device=DEVICE) * slot
        self.used = torch.zeros(S, dtype=torch.int32, device=DEVICE)
        self.slot = slot

    def append(self, k, v):
        """One token of every sequence."""
        at = (self.first[:-1] + self.used).long()
        self.k[at], self.v[at] = k, v
        self.used += 1


def next_tokens(qkv, weights, cache, Hq, Hkv, workspace=None):
    """qkv: [S, 1, Hq + 2 Hkv, D], the next token of every sequence.  Returns the attention's output [S, Hq, D]."""
    S, _, _, D = qkv.shape
    heads = [Hq, Hkv, Hkv]
    rotary = prompt_rotary(D, cache.used[:, None].clone())
    rows = [torch.empty((S, 1, h, D), dtype=BF16, device=DEVICE) for h in heads]
    sta.sta_qk_norm_rope(*qkv.split(heads, 2), *rows, *weights, rotary)
    q, k, v = (r[:, 0] for r in rows)
    cache.append(k, v)
    o = torch.empty_like(q)
    if workspace is None:
        workspace = scratch(sta.sta_packed_workspace_bytes(Hq, Hkv, D, S, S, 1, cache.slot))
    sta.sta_packed_forward(q, cache.k, cache.v, o, torch.arange(S + 1, dtype=torch.int32, device=DEVICE), cache.first, 1, cache.slot,
                           k_used=cache.used, workspace=workspace)
    return o


class PagedCache:
    """Two pools of pages, one that is used and one that keys are taken over to when there are too many; every sequence has as many pages in either."""

    def __init__(self, S, room, page, Hkv, D):
        n = -(-room // page)
        self.caches, self.weights, self.now = [], [], 0
        for _ in range(2):
            k, v = torch.zeros((2, S * n, page, Hkv, D), dtype=BF16, device=DEVICE)
            table = torch.randperm(S * n, device=DEVICE).to(torch.int32).view(S, n)      # any pages that are free
            self.caches.append(sta.StaPagedCache(k, v, table, torch.zeros(S, dtype=torch.int32, device=DEVICE)))
            self.weights.append(torch.zeros((S * n, Hkv, page), device=DEVICE))

    def step(self, q, k, v, lengths, longest, window):
        """New rows into their pages, attention over them, and what the last `window` tokens of every sequence look at, added to what its keys have gathered.  longest: no sequence has
        more keys.  Returns the attention's output."""
        cache, weights, cu = self.caches[self.now], self.weights[self.now], starts(lengths)
        Hq, most = q.shape[1], max(lengths)
        cache.used.add_(torch.tensor(lengths, dtype=torch.int32, device=DEVICE))
        sta.sta_paged_append(k, v, cu, cache, most, weights=weights)
        o, lse = torch.empty_like(q), torch.empty((Hq, q.shape[0]), device=DEVICE)
        workspace = scratch(sta.sta_paged_workspace_bytes(Hq, k.shape[1], q.shape[2], cache.S, q.shape[0], most, longest))
        sta.sta_paged_forward(q, o, cu, cache, most, longest, lse=lse, workspace=workspace)
        if most > window:
            ends, last = [sum(lengths[:i + 1]) for i in range(len(lengths))], [min(n, window) for n in lengths]
            rows = torch.cat([torch.arange(e - n, e, device=DEVICE) for e, n in zip(ends, last)])
            q, lse, cu, most = q[rows], lse[:, rows].contiguous(), starts(last), max(last)
        sta.sta_paged_weights(q, lse, weights, cu, cache, most, longest, before=weights)
        return o

    def cut(self, keep, first, recent):
        """Leaves every sequence at most `keep` keys.  Returns which they were, [S, Hkv, keep]."""
        old, new = self.caches[self.now], self.caches[1 - self.now]
        kept = torch.empty((old.S, old.Hkv, keep), dtype=torch.int32, device=DEVICE)
        sta.sta_paged_evict(old, self.weights[self.now], new, self.weights[1 - self.now], kept, first=first, recent=recent)
        self.now = 1 - self.now
        return kept


def conversation(qkv, further, weights, lengths, Hq, Hkv, keep, page=16, window=32):
    """qkv: [1, tokens, Hq + 2 Hkv, D], prompt after prompt; further: [steps, S, Hq + 2 Hkv, D], the next tokens of every prompt.  The prompts' keys are cut to `keep` by what the
    prompts' last tokens look at, then the next tokens go on.  Returns the prompts' output, which keys stayed, and the next tokens' outputs."""
    _, T, _, D = qkv.shape
    S, steps, heads = len(lengths), further.shape[0], [Hq, Hkv, Hkv]
    cache = PagedCache(S, max(lengths) + steps, page, Hkv, D)

    def rows_of(x, positions):
        out = [torch.empty((1, x.shape[1], h, D), dtype=BF16, device=DEVICE) for h in heads]
        sta.sta_qk_norm_rope(*x.split(heads, 2), *out, *weights, prompt_rotary(D, positions))
        return [r[0] for r in out]

    q, k, v = rows_of(qkv, torch.cat([torch.arange(n, dtype=torch.int32) for n in lengths]).to(DEVICE))
    o = cache.step(q, k, v, lengths, max(lengths), window)
    kept = cache.cut(keep, 4, keep // 4)
    outs = []
    for i, x in enumerate(further):             # positions go on from the whole prompts: rotations tell the keys that stayed where they stood
        q, k, v = rows_of(x[None], torch.tensor(lengths, dtype=torch.int32, device=DEVICE) + i)
        outs.append(cache.step(q, k, v, [1] * S, max(lengths) + i + 1, 1))
    return o, kept, outs


def main(grid=(6, 16, 24), tile=(6, 8, 8), H=4, Hq=8, Hkv=2, D=128, lengths=(300, 41, 1)):
    g = torch.Generator(device=DEVICE).manual_seed(0)

    def randn(*shape, dtype=BF16):
        return torch.randn(shape, generator=g, device=DEVICE).to(dtype)

    weights = [1.0 + 0.1 * randn(D, dtype=torch.float32) for _ in range(2)]
    N = grid[0] * grid[1] * grid[2]
    o, d_qkv, _ = video_layer(randn(1, N, 3 * H, D), randn(1, H, N, D), weights, grid, tile, [(1, 3, 3)] * H)
    print("video layer: output %s, gradient of the projection's output %s" % (tuple(o.shape), tuple(d_qkv.shape)))

    lengths, T = list(lengths), sum(lengths)
    qkv = randn(1, T, Hq + 2 * Hkv, D)
    o, k, v, d_qkv, _ = prompt_layer(qkv, randn(T, Hq, D), weights, lengths, Hq, Hkv)
    print("prompts of %s tokens: output %s, gradient of the projection's output %s" % (lengths, tuple(o.shape), tuple(d_qkv.shape)))

    # the last token of every prompt once more, as a next token against the others' keys and values
    cache = Cache(len(lengths), max(lengths) + 8, Hkv, D)
    first = [sum(lengths[:i]) for i in range(len(lengths))]
    for s, (a, n) in enumerate(zip(first, lengths)):
        cache.k[s * cache.slot:s * cache.slot + n - 1], cache.v[s * cache.slot:s * cache.slot + n - 1] = k[a:a + n - 1], v[a:a + n - 1]
        cache.used[s] = n - 1
    last = torch.tensor([a + n - 1 for a, n in zip(first, lengths)], device=DEVICE)
    again = next_tokens(qkv[0, last][:, None], weights, cache, Hq, Hkv)
    error = float((again.float() - o[last].float()).norm() / o[last].float().norm())
    print("next tokens against a cache of %d of %d slots: off the prompts' last rows by %.1e (2-norm)" % (int(cache.used.sum()), cache.k.shape[0], error))

    steps, keep = 5, 64
    o, kept, outs = conversation(qkv, randn(steps, len(lengths), Hq + 2 * Hkv, D), weights, lengths, Hq, Hkv, keep)
    print("conversations of %s tokens cut to %s keys: output of the prompts %s, of %d tokens each %s" % (
        lengths, [min(n, keep) for n in lengths], tuple(o.shape), steps, tuple(outs[-1].shape)))
    return error


if __name__ == "__main__":
    main()
