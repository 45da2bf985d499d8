"""What stands around the sliding tile attention in a transformer layer, as cases that can be timed and compared: the norms of
query and key heads with the rotation of positions and the move into tile order, the rotation alone, and attention over packed
sequences with grouped heads.  `own` chooses between the plain form, elementary torch operations in 32 bits, and the package's
own entry points.

A case is a dict of plain values.  "kind" is
  "norm_rope"   B, N or grid and tile ("TxHxW"), Hq, Hkv, D, rot (rotated channels), interleaved, f32 (inputs float32), train
  "rope"        B, N, Hq, Hkv, D, rot, interleaved, f32, scaling ("none", "linear", "ntk", "yarn"), factor, start, train
  "attention"   Hq, Hkv, D, lengths_q and lengths_k (comma-separated, one per sequence), causal, cache (slots of one size that hold
                the keys; 0: packed one behind the other), train
Training cases run the operator and its gradients.
"""
import math

import torch

own = False
DEVICE = "cuda:0"
EPS = 1e-6
THETA = 10000.0


def _norm_rope(B, Hq, Hkv, D, rot, interleaved, N=0, grid="", tile="", f32=False, train=False, name=None):
    case = {"kind": "norm_rope", "B": B, "N": N, "grid": grid, "tile": tile, "Hq": Hq, "Hkv": Hkv, "D": D, "rot": rot,
            "interleaved": interleaved, "f32": f32, "train": train}
    return dict(case, name=name) if name else case


def _rope(B, N, Hq, Hkv, D, rot, interleaved, scaling="none", factor=1.0, start=0, f32=False, train=False, name=None):
    case = {"kind": "rope", "B": B, "N": N, "Hq": Hq, "Hkv": Hkv, "D": D, "rot": rot, "interleaved": interleaved,
            "scaling": scaling, "factor": factor, "start": start, "f32": f32, "train": train}
    return dict(case, name=name) if name else case


def _attention(Hq, Hkv, D, lengths_q, lengths_k, causal=True, cache=0, train=False, name=None):
    case = {"kind": "attention", "Hq": Hq, "Hkv": Hkv, "D": D, "lengths_q": ",".join(str(x) for x in lengths_q),
            "lengths_k": ",".join(str(x) for x in lengths_k), "causal": causal, "cache": cache, "train": train}
    return dict(case, name=name) if name else case


def listed():
    decoded = [1 + (7919 * i) % 16384 for i in range(48)]
    packed = [2048, 1999, 77, 1023, 949]
    return [
        # The next token of four sequences: latency.
        _norm_rope(4, 32, 8, 128, 128, False, N=1, name="norm_rope_tokens"),
        # A prompt of an odd length, half of every head rotated.
        _norm_rope(1, 32, 8, 128, 64, False, N=4099, name="norm_rope_prompt"),
        # The video latent of the sliding tile attention's headline layer, from the projection into tile order.
        _norm_rope(1, 24, 24, 128, 128, True, grid="30x48x80", tile="6x8x8", name="norm_rope_video"),
        # Finetuning on short clips: forward and gradients, float32 activations.
        _norm_rope(1, 12, 12, 128, 128, True, grid="12x48x48", tile="6x8x8", f32=True, train=True, name="norm_rope_train_clip"),
        # A long context whose frequencies are scaled, its positions far from zero.
        _rope(1, 32768, 32, 8, 128, 128, False, scaling="yarn", factor=8.0, start=98304, name="rope_long"),
        # A ragged batch of a small model with odd heads: part of the head, neighbouring channels, both directions.
        _rope(7, 333, 5, 5, 80, 40, True, f32=True, train=True, name="rope_train_small"),
        # Three short captions, every token seeing its whole caption: latency.
        _attention(12, 12, 64, [77, 12, 1], [77, 12, 1], causal=False, name="attention_captions"),
        # Two long prompts of different lengths, packed.
        _attention(32, 8, 128, [8192, 4097], [8192, 4097], name="attention_prompts"),
        # 256 further tokens of two long conversations whose keys are in a cache.
        _attention(32, 8, 128, [256, 256], [32768, 20001], cache=32768, name="attention_chunk"),
        # The next token of 48 conversations.
        _attention(32, 8, 128, [1] * 48, decoded, cache=16384, name="attention_tokens"),
        # Training on packed documents with grouped heads.
        _attention(32, 8, 128, packed, packed, train=True, name="attention_train"),
        # Training on captions with a small head dimension, one head of keys for each head of queries.
        _attention(16, 16, 64, [333, 1024, 65, 2048, 578], [333, 1024, 65, 2048, 578], train=True, name="attention_train_d64"),
    ]


def _log_uniform(rng, lo, hi):
    return math.exp(rng.uniform(math.log(lo), math.log(hi)))


def _log_int(rng, lo, hi):
    return max(lo, min(hi, round(_log_uniform(rng, lo, hi))))


def _heads(rng):
    Hkv = rng.choice([1, 2, 3, 4, 5, 8, 8, 12])
    group = rng.choice([1, 1, 2, 4, 4, 5, 8])
    return min(Hkv * group, 40) // Hkv * Hkv, Hkv


def _rotated(rng, D):
    return rng.choice([D, D, D, D // 2, D // 4])


def draw(rng):
    kind = rng.choice(["norm_rope", "norm_rope", "rope", "attention", "attention", "attention"])
    train = rng.random() < 0.4
    if kind == "norm_rope":
        if rng.random() < 0.5:          # a video or image latent, into tile order
            tile = rng.choice([(6, 8, 8), (1, 8, 8), (2, 8, 8), (2, 6, 8), (4, 4, 8)])
            D, H = rng.choice([64, 128]), rng.choice([1, 3, 5, 8, 12, 24])
            tiles = _log_uniform(rng, 2, min(300, 115200 / (tile[0] * tile[1] * tile[2])))
            n_t = 1 if tile[0] == 1 else max(1, min(5, round(tiles ** (1 / 3) * rng.uniform(0.4, 1.2))))
            n_h = max(1, int(math.sqrt(tiles / n_t)))
            n_w = max(1, int(tiles / (n_t * n_h)))
            grid = "%dx%dx%d" % (n_t * tile[0], n_h * tile[1], n_w * tile[2])
            f32 = rng.random() < 0.3 and H <= 12
            return _norm_rope(1 if H > 8 else rng.randint(1, 2), H, H, D, D, rng.random() < 0.7, grid=grid,
                              tile="%dx%dx%d" % tile, f32=f32, train=train and H <= 12)
        Hq, Hkv = _heads(rng)
        D = rng.choice([64, 80, 96, 128, 128, 256])
        B = rng.choice([1, 1, 2, 5])
        return _norm_rope(B, Hq, Hkv, D, _rotated(rng, D), rng.random() < 0.4, N=_log_int(rng, 1, 8192 // B), f32=rng.random() < 0.3,
                          train=train)
    if kind == "rope":
        Hq, Hkv = _heads(rng)
        D = rng.choice([64, 80, 96, 128, 128, 256])
        scaling = rng.choice(["none", "linear", "ntk", "yarn"])
        B = rng.choice([1, 1, 3, 8])
        return _rope(B, _log_int(rng, 1, 8192 // B), Hq, Hkv, D, _rotated(rng, D), rng.random() < 0.4, scaling=scaling,
                     factor=1.0 if scaling == "none" else rng.choice([2.0, 4.0, 8.0, 2.5]), start=_log_int(rng, 1, 1000000) - 1,
                     f32=rng.random() < 0.3, train=train)
    form = "train" if train else rng.choice(["prompts", "prompts", "chunk", "tokens"])
    while True:
        Hq, Hkv = _heads(rng)
        D = rng.choice([64, 128, 128])
        if form in ("train", "prompts"):
            budget, longest = _log_int(rng, 8, 12288), _log_int(rng, 8, 8192)
            queries = []
            while budget > 0 and len(queries) < 40:
                queries.append(min(budget, _log_int(rng, 1, longest)))
                budget -= queries[-1]
            keys = queries
            if rng.random() < 0.25:         # keys and queries of different numbers: a causal row may then see none
                keys = [max(1, round(x * rng.uniform(0.5, 1.5))) for x in queries]
        else:
            S = _log_int(rng, 1, 64 if form == "tokens" else 6)
            most = _log_int(rng, 32, 16384 if form == "tokens" else 32768)
            keys = [rng.randint(1, most) for _ in range(S)]
            queries = [rng.choice([1, 1, 1, 2, 4])] * S if form == "tokens" else [_log_int(rng, 1, 512) for _ in range(S)]
            keys = [max(a, b) for a, b in zip(queries, keys)]
        # scores of sequences filled up to the longest one, which the plain form holds
        if len(keys) * max(queries) * max(keys) * Hq <= (2 ** 30 if form == "train" else 2 ** 32):
            cache = 0 if form in ("train", "prompts") else max(keys)
            causal = cache > 0 or rng.random() < 0.75
            return _attention(Hq, Hkv, D, queries, keys, causal=causal, cache=cache, train=form == "train")


def _triple(text):
    return tuple(int(x) for x in text.split("x"))


def _lengths(text):
    return [int(x) for x in text.split(",")]


class _State:
    pass


def prepare(case, seed):
    generator = torch.Generator(device=DEVICE)
    generator.manual_seed(seed)

    def normal(*shape, dtype=torch.bfloat16, spread=1.0):
        return (torch.randn(shape, generator=generator, dtype=torch.float32, device=DEVICE) * spread).to(dtype)

    def ints(values, dtype=torch.int32):
        return torch.tensor(values, dtype=dtype, device=DEVICE)

    s = _State()
    s.kind, s.train = case["kind"], case["train"]
    Hq, Hkv, D = case["Hq"], case["Hkv"], case["D"]
    if s.kind == "attention":
        lq, lk, s.causal, s.cache = _lengths(case["lengths_q"]), _lengths(case["lengths_k"]), case["causal"], case["cache"]
        S, tq = len(lq), sum(lq)
        tk = S * s.cache if s.cache else sum(lk)
        # activations behind a norm
        s.q, s.k, s.v = normal(tq, Hq, D), normal(tk, Hkv, D), normal(tk, Hkv, D)
        s.d_o = normal(tq, Hq, D) if s.train else None
        s.max_q, s.max_k, s.scale = max(lq), max(lk), D ** -0.5
        s.len_q, s.len_k = ints(lq), ints(lk)
        slots = [s.cache] * S if s.cache else lk
        s.cu_q, s.cu_k = (ints([sum(x[:i]) for i in range(S + 1)]) for x in (lq, slots))
        s.k_used = s.len_k if s.cache else None
        s.lse = torch.empty((Hq, tq), dtype=torch.float32, device=DEVICE) if s.train else None
        s.out = [torch.empty_like(x) for x in ((s.q, s.q, s.k, s.v) if s.train else (s.q,))]
        if own:
            import paper_2502_04507_amd as sta
            need = sta.sta_packed_backward_workspace_bytes(Hq, tq) if s.train else \
                sta.sta_packed_workspace_bytes(Hq, Hkv, D, S, tq, s.max_q, s.max_k)
            s.workspace = torch.empty(max(16, need), dtype=torch.uint8, device=DEVICE)
        return s

    B, s.rot, s.interleaved = case["B"], case["rot"], case["interleaved"]
    dtype = torch.float32 if case["f32"] else torch.bfloat16
    normed = s.kind == "norm_rope"
    s.grid, s.tile = (_triple(case["grid"]), _triple(case["tile"])) if normed and case["grid"] else (None, None)
    N = s.grid[0] * s.grid[1] * s.grid[2] if s.grid else case["N"]
    heads = [Hq, Hkv, Hkv] if normed else [Hq, Hkv]
    # What the projection leaves, token after token: query, key and value heads.
    x = normal(B, N, sum(heads), D, dtype=dtype, spread=2.0)
    s.x = list(x.split(heads, 2))
    s.weights = [1.0 + normal(D, dtype=torch.float32, spread=0.2) for _ in range(2)] if normed else None

    # Rotated pairs of every axis: all of them, or for a video an eighth for time and the rest in equal parts for height and width.
    pairs, side = s.rot // 2, s.rot * 7 // 32
    s.pairs = (pairs - 2 * side, side, side) if s.grid else (pairs,)
    # Turns per position in units of 2^-64, and the factor on the rotated channels.
    scaling, factor = (case["scaling"], case["factor"]) if s.kind == "rope" else ("none", 1.0)
    s.magnitude = 0.1 * math.log(factor) + 1.0 if scaling == "yarn" else 1.0
    steps, s.axis = [], []
    for axis, n in enumerate(s.pairs):
        base = THETA * factor ** (n / (n - 1.0)) if scaling == "ntk" and n > 1 else THETA
        for i in range(n):
            f = base ** (-i / n) / (factor if scaling == "linear" else 1.0)
            if scaling == "yarn":
                keep = min(1.0, max(0.0, (4096 * f / (2 * math.pi) - 1.0) / (32.0 - 1.0)))
                f = f * keep + f / factor * (1.0 - keep)
            step = round(f / (2 * math.pi) * 2.0 ** 64)
            steps.append(step - 2 ** 64 if step >= 2 ** 63 else step)
            s.axis.append(axis)
    s.steps, s.axis = ints(steps, torch.int64), ints(s.axis, torch.int64)
    if s.grid:
        t, h, w = (torch.arange(n, dtype=torch.int32, device=DEVICE) for n in s.grid)
        s.positions = torch.stack(torch.meshgrid(t, h, w, indexing="ij"), -1).reshape(N, 3)
    else:
        start = case["start"] if s.kind == "rope" else 17
        s.positions = torch.arange(start, start + N, dtype=torch.int32, device=DEVICE)[:, None]
    s.out_type = torch.bfloat16 if s.tile else dtype            # the sliding tile attention reads bfloat16
    # Outputs, and their gradients as they come back, in tile order head by head, or else token after token.
    order = [(B, h, N, D) if s.tile else (B, N, h, D) for h in heads]
    s.out = [torch.empty(o, dtype=s.out_type, device=DEVICE) for o in order]
    s.d_out = [normal(*o, dtype=s.out_type) for o in order] if s.train else []
    if s.tile:
        s.out, s.d_out = ([t.transpose(1, 2) for t in ts] for ts in (s.out, s.d_out))
    if s.train:
        s.d = list(torch.empty_like(x).split(heads, 2))         # what the projection's gradient reads
        s.d_weights = [torch.empty(D, dtype=torch.float32, device=DEVICE) for _ in range(2)] if normed else []
    if own:
        import paper_2502_04507_amd as sta
        s.rotary = sta.StaRotary(s.steps, positions=None if s.grid else s.positions[:, 0], pairs=s.pairs, interleaved=s.interleaved,
                                 magnitude=s.magnitude)
        if s.train and normed:
            s.workspace = torch.empty(max(16, sta.sta_qk_norm_rope_workspace_bytes(D)), dtype=torch.uint8, device=DEVICE)
    return s


# ---- the plain form: elementary operations in 32 bits ------------------------------------------------------------------------
def _turns(s):
    """Cosines and sines of every token and pair, [N, 1, rot / 2], times the magnitude."""
    phase = s.positions.to(torch.int64)[:, s.axis] * s.steps          # turns in units of 2^-64, modulo whole turns
    angle = (phase.to(torch.float32) * (2.0 * math.pi * 2.0 ** -64))[:, None]
    return torch.cos(angle) * s.magnitude, torch.sin(angle) * s.magnitude


def _rotate(s, x, cos, sin):
    rotated = x[..., :s.rot]
    if s.interleaved:
        a, b = rotated[..., 0::2], rotated[..., 1::2]
        y = torch.stack((a * cos - b * sin, a * sin + b * cos), -1).flatten(-2)
    else:
        a, b = rotated[..., :s.rot // 2], rotated[..., s.rot // 2:]
        y = torch.cat((a * cos - b * sin, a * sin + b * cos), -1)
    return y if s.rot == x.shape[-1] else torch.cat((y, x[..., s.rot:]), -1)


def _tiles(s, x):
    """Tokens in raster order, [B, N, H, D], into tile order head by head."""
    B, N, H, D = x.shape
    (gt, gh, gw), (t, h, w) = s.grid, s.tile
    x = x.view(B, gt // t, t, gh // h, h, gw // w, w, H, D).permute(0, 7, 1, 3, 5, 2, 4, 6, 8)
    return x.reshape(B, H, N, D).transpose(1, 2)


def _raster(s, x):
    B, N, H, D = x.shape
    (gt, gh, gw), (t, h, w) = s.grid, s.tile
    x = x.transpose(1, 2).reshape(B, H, gt // t, gh // h, gw // w, t, h, w, D).permute(0, 2, 5, 3, 6, 4, 7, 1, 8)
    return x.reshape(B, N, H, D)


def _plain_norm_rope(s):
    cos, sin = _turns(s)
    place = (lambda x: _tiles(s, x.to(s.out_type))) if s.tile else (lambda x: x.to(s.out_type))
    back = (lambda d: _raster(s, d).float()) if s.tile else (lambda d: d.float())

    def forward(x, w):
        x = x.float()
        return place(_rotate(s, x * torch.rsqrt((x * x).mean(-1, keepdim=True) + EPS) * w, cos, sin))

    def backward(x, w, d):
        x = x.float()
        r = torch.rsqrt((x * x).mean(-1, keepdim=True) + EPS)
        g = _rotate(s, back(d), cos, -sin)
        gw = g * w
        return (r * (gw - x * (r * r * (gw * x).mean(-1, keepdim=True)))).to(s.x[0].dtype), (g * x * r).sum((0, 1, 2))

    q, k, v = s.x
    out = [forward(q, s.weights[0]), forward(k, s.weights[1]), place(v)]
    if not s.train:
        return out
    (d_q, d_wq), (d_k, d_wk) = backward(q, s.weights[0], s.d_out[0]), backward(k, s.weights[1], s.d_out[1])
    return out + [d_q, d_k, back(s.d_out[2]).to(v.dtype), d_wq, d_wk]


def _plain_rope(s):
    cos, sin = _turns(s)
    out = [_rotate(s, x.float(), cos, sin).to(x.dtype) for x in s.x]
    return out + [_rotate(s, d.float(), cos, -sin).to(d.dtype) for d in s.d_out]


def _plain_attention(s):
    """All sequences at once, each filled up to the longest one."""
    (tq, Hq, D), Hkv, S = s.q.shape, s.k.shape[1], s.len_q.shape[0]
    i, j = (torch.arange(n, device=DEVICE) for n in (s.max_q, s.max_k))

    def filled(x, cu, place):           # [S, heads, longest, D]
        at = (cu[:-1, None] + place).clamp(max=x.shape[0] - 1)
        return x[at].float().transpose(1, 2).contiguous()

    def packed(x, cu, tokens):          # back to [tokens, heads, D]
        n = torch.arange(tokens, device=DEVICE)
        seq = torch.searchsorted(cu[1:], n, right=True)
        return x[seq, :, n - cu[seq]]

    q = filled(s.q, s.cu_q, i).view(S, Hkv, Hq // Hkv * s.max_q, D)
    k, v = filled(s.k, s.cu_k, j), filled(s.v, s.cu_k, j)
    keep = (j < s.len_k[:, None])[:, None, None, None, :]
    if s.causal:
        keep = keep & (j <= i[:, None] + (s.len_k - s.len_q)[:, None, None])[:, None, None]
    scores = (torch.matmul(q, k.transpose(2, 3).contiguous()) * s.scale).view(S, Hkv, Hq // Hkv, s.max_q, s.max_k)
    scores = scores.masked_fill(~keep, -math.inf).view(S, Hkv, -1, s.max_k)
    top = scores.max(-1, keepdim=True).values
    top = torch.where(torch.isinf(top), 0.0, top)
    p = torch.exp(scores - top)
    del scores
    total = p.sum(-1, keepdim=True)
    p = p / torch.where(total > 0, total, 1.0)
    y = torch.matmul(p, v)
    o = packed(y.view(S, Hq, s.max_q, D), s.cu_q, tq).to(s.q.dtype)
    if not s.train:
        return [o]
    lse = packed((top + torch.log(total)).view(S, Hq, s.max_q, 1), s.cu_q, tq)[..., 0].t().contiguous()
    inside = (i < s.len_q[:, None])[:, None, :, None]
    d_o = (filled(s.d_o, s.cu_q, i) * inside).view(S, Hkv, -1, D)
    d_v = torch.matmul(p.transpose(2, 3).contiguous(), d_o)
    d_s = p * (torch.matmul(d_o, v.transpose(2, 3).contiguous()) - (d_o * y).sum(-1, keepdim=True)) * s.scale
    d_q = torch.matmul(d_s, k).view(S, Hq, s.max_q, D)
    d_k = torch.matmul(d_s.transpose(2, 3).contiguous(), q)
    tk = s.k.shape[0]
    return [o, lse, packed(d_q, s.cu_q, tq).to(o.dtype), packed(d_k, s.cu_k, tk).to(o.dtype), packed(d_v, s.cu_k, tk).to(o.dtype)]


# ---- the package's operators ---------------------------------------------------------------------------------------------------
def _own(s):
    import paper_2502_04507_amd as sta
    if s.kind == "norm_rope":
        sta.sta_qk_norm_rope(*s.x, *s.out, *s.weights, s.rotary, eps=EPS, grid=s.grid, tile=s.tile)
        if not s.train:
            return s.out
        sta.sta_qk_norm_rope_backward(s.x[0], s.x[1], *s.d_out, *s.d, *s.weights, *s.d_weights, s.rotary, s.workspace, eps=EPS,
                                      grid=s.grid, tile=s.tile)
        return s.out + s.d + s.d_weights
    if s.kind == "rope":
        sta.sta_rope(s.x, s.out, s.rotary)
        if not s.train:
            return s.out
        sta.sta_rope(s.d_out, s.d, s.rotary, inverse=True)
        return s.out + s.d
    if not s.train:
        sta.sta_packed_forward(s.q, s.k, s.v, s.out[0], s.cu_q, s.cu_k, s.max_q, s.max_k, causal=s.causal, k_used=s.k_used,
                               workspace=s.workspace)
        return s.out
    o, *d = s.out
    sta.sta_packed_forward(s.q, s.k, s.v, o, s.cu_q, s.cu_k, s.max_q, s.max_k, causal=s.causal, lse=s.lse)
    sta.sta_packed_backward(s.q, s.k, s.v, o, s.d_o, s.lse, *d, s.cu_q, s.cu_k, s.max_q, s.max_k, s.workspace, causal=s.causal)
    return [o, s.lse] + d


def run(s):
    if own:
        return _own(s)
    if s.kind == "norm_rope":
        return _plain_norm_rope(s)
    return _plain_rope(s) if s.kind == "rope" else _plain_attention(s)


# ---- the definitions in 64 bits ------------------------------------------------------------------------------------------------
def exact(case, seed):
    s = prepare(case, seed)
    if case["kind"] == "attention":             # one sequence and head after the other
        Hq, Hkv, D = case["Hq"], case["Hkv"], case["D"]
        group = Hq // Hkv
        o = torch.zeros(s.q.shape, dtype=torch.float64, device=DEVICE)
        lse = torch.full((Hq, s.q.shape[0]), -math.inf, dtype=torch.float64, device=DEVICE)
        d_q = torch.zeros_like(o)
        d_k, d_v = (torch.zeros(s.k.shape if s.train else (1,), dtype=torch.float64, device=DEVICE) for _ in range(2))
        cu_q, cu_k = s.cu_q.tolist(), s.cu_k.tolist()
        for n, (lq, lk) in enumerate(zip(_lengths(case["lengths_q"]), _lengths(case["lengths_k"]))):
            rows, keys = slice(cu_q[n], cu_q[n] + lq), slice(cu_k[n], cu_k[n] + lk)
            for h in range(Hq):
                q, k, v = s.q[rows, h].double(), s.k[keys, h // group].double(), s.v[keys, h // group].double()
                scores = q @ k.T / math.sqrt(D)
                if s.causal:
                    scores += torch.full_like(scores, -math.inf).triu(lk - lq + 1)
                z = torch.logsumexp(scores, -1)
                p = torch.exp(scores - z[:, None]).nan_to_num(0.0)
                o[rows, h], lse[h, rows] = p @ v, z
                if s.train:
                    g = s.d_o[rows, h].double()
                    d_v[keys, h // group] += p.T @ g
                    d_p = g @ v.T
                    d_s = p * (d_p - (p * d_p).sum(-1, keepdim=True)) / math.sqrt(D)
                    d_q[rows, h] = d_s @ k
                    d_k[keys, h // group] += d_s.T @ q
        return [o, lse, d_q, d_k, d_v] if s.train else [o]

    # pairs as complex numbers: times exp(i angle), their gradients times exp(-i angle)
    angle = (s.positions.long()[:, s.axis] * s.steps).double() / 2.0 ** 63 * math.pi
    turn = torch.polar(torch.full_like(angle, s.magnitude), angle)[None, :, None, :]
    first = slice(0, s.rot, 2) if s.interleaved else slice(0, s.rot // 2)
    second = slice(1, s.rot, 2) if s.interleaved else slice(s.rot // 2, s.rot)

    def rotated(x, by):
        y = x.clone()
        z = torch.complex(x[..., first].contiguous(), x[..., second].contiguous()) * by
        y[..., first], y[..., second] = z.real, z.imag
        return y

    if s.kind == "rope":
        return [rotated(x.double(), turn) for x in s.x] + [rotated(d.double(), turn.conj()) for d in s.d_out]
    if s.tile:
        (_, gh, gw), (tt, th, tw) = s.grid, s.tile
        p = s.positions.long()
        tile = ((p[:, 0] // tt) * (gh // th) + p[:, 1] // th) * (gw // tw) + p[:, 2] // tw
        place = tile * (tt * th * tw) + ((p[:, 0] % tt) * th + p[:, 1] % th) * tw + p[:, 2] % tw
        order = torch.argsort(place)                            # raster index of the token at every place
    out, grads, d_weights = [], [], []
    for n, x in enumerate(s.x):
        x, g = x.double(), s.d_out[n].double() if s.train else None
        if s.train and s.tile:
            g = g[:, place]
        y = x
        if n < 2:
            rms = (x.square().sum(-1, keepdim=True) / case["D"] + EPS).sqrt()
            unit, w = x / rms, s.weights[n].double()
            y = rotated(unit * w, turn)
            if s.train:
                g = rotated(g, turn.conj())
                d_weights.append((g * unit).sum(dim=(0, 1, 2)))
                g = g * w
                g = (g - unit * ((g * unit).sum(-1, keepdim=True) / case["D"])) / rms
        out.append(y[:, order] if s.tile else y)
        grads.append(g)
    return out + grads + d_weights if s.train else out


def _seen(lq, lk, causal):
    """Pairs of a row and a key that it sees."""
    if not causal:
        return lq * lk
    rows = min(lq, lk)                     # the rows that see a key: the last lk ones see 1 .. lk, or the first sees lk - lq + 1
    first = lk - rows + 1
    return rows * (first + lk) // 2


def work(case):
    Hq, Hkv, D = case["Hq"], case["Hkv"], case["D"]
    if case["kind"] == "attention":
        lq, lk = _lengths(case["lengths_q"]), _lengths(case["lengths_k"])
        rows, keys = sum(lq) * Hq * D * 2, sum(lk) * Hkv * D * 2
        flops = 4.0 * D * Hq * sum(_seen(a, b, case["causal"]) for a, b in zip(lq, lk))
        if not case["train"]:
            return {"bytes": 2 * rows + 2 * keys, "flops": flops}
        return {"bytes": 4 * rows + 4 * keys + 4 * Hq * sum(lq), "flops": 3.5 * flops}     # five more products
    size = 4 if case["f32"] else 2
    if case["kind"] == "rope":
        elements = case["B"] * case["N"] * (Hq + Hkv) * D
        passes = 2 if case["train"] else 1
        return {"bytes": passes * 2 * size * elements, "flops": passes * 3.0 * elements * case["rot"] / D}
    grid = _triple(case["grid"]) if case["grid"] else (1, 1, case["N"])
    tokens = case["B"] * grid[0] * grid[1] * grid[2]
    elements, normed = tokens * (Hq + 2 * Hkv) * D, tokens * (Hq + Hkv) * D
    out = 2 if case["tile"] else size
    if not case["train"]:
        return {"bytes": elements * (size + out), "flops": 7.0 * normed}
    # the forward's inputs are read once for both directions
    return {"bytes": elements * 2 * (size + out), "flops": 22.0 * normed}
