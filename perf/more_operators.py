"""A cache of keys and values in pages and what works on it, as cases that can be timed and compared: new rows written into their pages,
attention of chunks of new tokens and of single tokens over the pages, the attention weight that every key has gathered, and the eviction of the
keys that gathered least.  `own` chooses between the plain form, elementary torch operations in 32 bits, and the package's own entry points.

Key j of sequence s is slot j % page of page table[s, j // page] of the pools k, v [pages, page, Hkv, D]; its weight for key head n is
weights[that page, n, that slot].

A case is a dict of plain values.  "kind" is
  "append"      Hkv, D, page, new and used (comma-separated, one per sequence: new tokens, and keys with them), f32 (rows float32)
  "attention"   Hq, Hkv, D, page, new, used, causal, lse (the rows' log sums are wanted too)
  "weights"     Hq, Hkv, D, page, new, used, decay (0: the rows' weights alone, nothing before them counts)
  "evict"       Hkv, D, page, used, keep, first, recent
"""
import math

import torch

own = False
DEVICE = "cuda:0"


def _text(values):
    return ",".join(str(x) for x in values)


def _case(kind, name, **rest):
    case = dict(kind=kind, **{k: _text(v) if isinstance(v, list) else v for k, v in rest.items()})
    return dict(case, name=name) if name else case


def _append(Hkv, D, page, new, used, f32=False, name=None):
    return _case("append", name, Hkv=Hkv, D=D, page=page, new=new, used=used, f32=f32)


def _attention(Hq, Hkv, D, page, new, used, causal=True, lse=False, name=None):
    return _case("attention", name, Hq=Hq, Hkv=Hkv, D=D, page=page, new=new, used=used, causal=causal, lse=lse)


def _weights(Hq, Hkv, D, page, new, used, decay=1.0, name=None):
    return _case("weights", name, Hq=Hq, Hkv=Hkv, D=D, page=page, new=new, used=used, decay=decay)


def _evict(Hkv, D, page, used, keep, first, recent, name=None):
    return _case("evict", name, Hkv=Hkv, D=D, page=page, used=used, keep=keep, first=first, recent=recent)


def listed():
    decoded = [1 + (7919 * i) % 16384 for i in range(48)]
    return [
        # The rows of the next token of 48 conversations: latency.
        _append(8, 128, 16, [1] * 48, [1 + (791 * i) % 1024 for i in range(48)], name="append_tokens"),
        # Three prompts at once, of which the second goes on behind an earlier part; rows in float32 as a norm left them.
        _append(8, 128, 64, [8192, 4097, 77], [8192, 6001, 77], f32=True, name="append_prompts"),
        # The next token of three short captions: latency.
        _attention(12, 12, 64, 16, [1, 1, 1], [77, 12, 1], name="attention_captions"),
        # The next token of 48 conversations.
        _attention(32, 8, 128, 16, [1] * 48, decoded, name="attention_tokens"),
        # 256 further tokens of two long conversations, the log sums kept for the weights.
        _attention(32, 8, 128, 64, [256, 256], [32768, 20001], lse=True, name="attention_chunk"),
        # A step in which prompts begin, go on and give single tokens, with small heads and pages that are no power of two.
        _attention(15, 5, 64, 24, [333, 1, 2048, 65, 1, 578], [1333, 4097, 2048, 3001, 77, 578], name="attention_mixed"),
        # What the next token of 48 conversations gives to the keys, added to what they have.
        _weights(32, 8, 128, 16, [1] * 48, decoded, name="weights_tokens"),
        # A window of 32 rows at the end of a prompt and a long chunk, weighed by themselves: which keys the prompt can do without.
        _weights(32, 8, 128, 64, [32, 512], [32768, 20001], decay=0.0, name="weights_chunk"),
        # Short sequences of a small model, older weight counting less: latency.
        _weights(16, 16, 64, 8, [1, 5, 33], [333, 65, 578], decay=0.96875, name="weights_small"),
        # Three short sequences of which one already fits: latency.
        _evict(4, 64, 8, [333, 77, 578], 128, 4, 32, name="evict_small"),
        # A single long conversation cut to a quarter.
        _evict(8, 128, 64, [32768], 8192, 4, 256, name="evict_long"),
        # A batch of conversations cut to one budget, most of it for the keys of the greatest weight.
        _evict(8, 128, 16, [1 + (7919 * i) % 16384 for i in range(24)], 2048, 4, 64, name="evict_batch"),
    ]


def _log_int(rng, lo, hi):
    return max(lo, min(hi, round(math.exp(rng.uniform(math.log(lo), math.log(hi))))))


def draw(rng):
    kind = rng.choice(["append", "attention", "attention", "attention", "weights", "weights", "evict", "evict"])
    Hkv, D = rng.choice([1, 2, 3, 4, 5, 8, 8, 12]), rng.choice([64, 128, 128])
    Hq = min(Hkv * rng.choice([1, 1, 2, 4, 4, 5, 8]), 40) // Hkv * Hkv
    page = rng.choice([1, 8, 16, 16, 20, 24, 32, 64, 64, 128, 256])
    if kind == "append":
        S, most = _log_int(rng, 1, 64), _log_int(rng, 1, 4096)
        new = [rng.randint(1, most) if rng.random() < 0.9 else 1 for _ in range(S)]
        while sum(new) > 12000:
            new = [(x + 1) // 2 for x in new]
        earlier = _log_int(rng, 1, 512)
        return _append(Hkv, D, page, new, [x + rng.randint(0, earlier) for x in new], f32=rng.random() < 0.4)
    if kind == "evict":
        S, most = _log_int(rng, 1, 24), _log_int(rng, 64, 32768)
        used = [rng.randint(1, most) for _ in range(S)]
        while sum(used) > 180000:
            used = [(x + 1) // 2 for x in used]
        keep = _log_int(rng, 8, max(8, max(used) // 2))
        while keep * S > 49152:
            keep = (keep + 1) // 2
        first = rng.randint(0, min(16, keep // 4))
        return _evict(Hkv, D, page, used, keep, first, rng.randint(0, keep // 2))
    while True:
        tokens = rng.random() < 0.4
        S = _log_int(rng, 1, 64 if tokens else 6)
        most = _log_int(rng, 32, 16384 if tokens else 32768)
        used = [rng.randint(1, most) for _ in range(S)]
        new = [rng.choice([1, 1, 1, 2, 4])] * S if tokens else [_log_int(rng, 1, 512) for _ in range(S)]
        if not tokens and rng.random() < 0.3:       # prompts from their beginning
            new = [min(2048, x) for x in used]
        used = [max(a, b) for a, b in zip(new, used)]
        # scores of sequences filled up to the longest one, which the plain form holds
        if S * max(new) * max(used) * Hq <= 2 ** 29:
            if kind == "weights":
                return _weights(Hq, Hkv, D, page, new, used, decay=rng.choice([0.0, 1.0, 1.0, 0.96875]))
            return _attention(Hq, Hkv, D, page, new, used, causal=rng.random() < 0.85, lse=rng.random() < 0.4)


def _lengths(text):
    return [int(x) for x in text.split(",")]


class _State:
    pass


def prepare(case, seed):
    generator = torch.Generator(device=DEVICE)
    generator.manual_seed(seed)

    def normal(*shape, dtype=torch.bfloat16, spread=1.0):
        return (torch.randn(shape, generator=generator, dtype=torch.float32, device=DEVICE) * spread).to(dtype)

    def ints(values):
        return torch.tensor(values, dtype=torch.int32, device=DEVICE)

    def pages_of(lengths):
        """A table whose pages lie in the pool without order, as they were handed out, and how many pages there are."""
        need = [-(-x // s.page) for x in lengths]
        order = torch.randperm(sum(need), generator=generator, device=DEVICE).to(torch.int32)
        table = torch.zeros((len(need), max(need)), dtype=torch.int32, device=DEVICE)
        at = 0
        for i, n in enumerate(need):
            table[i, :n] = order[at:at + n]
            at += n
        return table, at

    s = _State()
    s.kind, s.Hkv, s.D, s.page = case["kind"], case["Hkv"], case["D"], case["page"]
    used = _lengths(case["used"])
    s.S, s.max_k, s.used = len(used), max(used), ints(used)
    s.table, pages = pages_of(used)
    s.k, s.v = normal(pages, s.page, s.Hkv, s.D), normal(pages, s.page, s.Hkv, s.D)
    if s.kind != "evict":
        new = _lengths(case["new"])
        s.max_q, tokens = max(new), sum(new)
        s.new, s.cu = ints(new), ints([sum(new[:i]) for i in range(len(new) + 1)])
    if s.kind == "append":
        # key and value heads as the projection leaves them, token after token
        rows = normal(tokens, 2 * s.Hkv, s.D, dtype=torch.float32 if case["f32"] else torch.bfloat16)
        s.k_new, s.v_new = rows.split(s.Hkv, 1)
        s.weights = normal(pages, s.Hkv, s.page, dtype=torch.float32).exp()
    if s.kind in ("attention", "weights"):
        s.Hq = case["Hq"]
        # scores of a spread of 2: some keys count for much more than others
        s.q, s.scale = normal(tokens, s.Hq, s.D, spread=2.0), s.D ** -0.5
        s.causal = case["causal"] if s.kind == "attention" else True
    if s.kind == "attention":
        s.o = torch.empty_like(s.q)
        s.lse = torch.empty((s.Hq, tokens), dtype=torch.float32, device=DEVICE) if case["lse"] else None
    if s.kind == "weights":
        s.decay = case["decay"]
        s.before = normal(pages, s.Hkv, s.page, dtype=torch.float32, spread=2.0).exp() if s.decay else None
        s.weights = torch.zeros((pages, s.Hkv, s.page), dtype=torch.float32, device=DEVICE)
        scores = _scores(s)
        top = scores.max(-1, keepdim=True).values
        s.lse = _packed(s, (top + torch.log(torch.exp(scores - top).sum(-1, keepdim=True))))[..., 0].t().contiguous()
        del scores
    if s.kind == "evict":
        s.keep, s.first, s.recent = case["keep"], case["first"], case["recent"]
        # a few keys have most of the weight, and some, such as new ones, none
        s.weights = normal(pages, s.Hkv, s.page, dtype=torch.float32, spread=2.0).exp()
        s.weights *= torch.rand(s.weights.shape, generator=generator, device=DEVICE) < 0.9
        s.to_table, to_pages = pages_of([min(s.keep, x) for x in used])
        if s.to_table.shape[1] * s.page < s.keep:       # room for as many keys as may stay
            s.to_table = torch.nn.functional.pad(s.to_table, (0, -(-s.keep // s.page) - s.to_table.shape[1]))
        s.to_k, s.to_v = (torch.zeros((to_pages, s.page, s.Hkv, s.D), dtype=torch.bfloat16, device=DEVICE) for _ in range(2))
        s.to_weights = torch.zeros((to_pages, s.Hkv, s.page), dtype=torch.float32, device=DEVICE)
        s.to_used = torch.zeros(s.S, dtype=torch.int32, device=DEVICE)
        s.kept = torch.empty((s.S, s.Hkv, s.keep), dtype=torch.int32, device=DEVICE)
    if own:
        import paper_2502_04507_amd as sta
        s.cache = sta.StaPagedCache(s.k, s.v, s.table, s.used)
        if s.kind == "evict":
            s.into = sta.StaPagedCache(s.to_k, s.to_v, s.to_table, s.to_used)
        if s.kind == "attention":
            need = sta.sta_paged_workspace_bytes(s.Hq, s.Hkv, s.D, s.S, s.q.shape[0], s.max_q, s.max_k)
            s.workspace = torch.empty(max(16, need), dtype=torch.uint8, device=DEVICE)
    return s


# ---- the plain form: elementary operations in 32 bits ------------------------------------------------------------------------
def _slots(s, table, j):
    """Places of keys j, [S, n], in a pool of pages laid side by side."""
    return torch.gather(table, 1, (j // s.page).clamp(max=table.shape[1] - 1)).long() * s.page + j % s.page


def _all_keys(s):
    return torch.arange(s.max_k, device=DEVICE).expand(s.S, -1)


def _key_rows(s, pool):
    """Rows of a pool, sequence by sequence and head by head, filled up to the longest: [S, Hkv, longest, D]."""
    return pool.view(-1, s.Hkv, s.D)[_slots(s, s.table, _all_keys(s))].float().transpose(1, 2).contiguous()


def _scores(s):
    """[S, Hkv, rows of the group, longest]; -infinity where a row does not see the key."""
    i, j = torch.arange(s.max_q, device=DEVICE), torch.arange(s.max_k, device=DEVICE)
    at = (s.cu[:-1, None] + i).clamp(max=s.q.shape[0] - 1)
    q = s.q[at].float().transpose(1, 2).reshape(s.S, s.Hkv, -1, s.D)
    scores = torch.matmul(q, _key_rows(s, s.k).transpose(2, 3).contiguous()) * s.scale
    sees = j < s.used[:, None, None]
    if s.causal:
        sees = sees & (j <= i[:, None] + (s.used - s.new)[:, None, None])
    scores = scores.view(s.S, s.Hkv, -1, s.max_q, s.max_k)
    return scores.masked_fill_(~sees[:, None, None], -math.inf).view(s.S, s.Hkv, -1, s.max_k)


def _packed(s, rows):
    """[S, Hkv, rows of the group, n] back to [tokens, Hq, n]."""
    n = torch.arange(s.q.shape[0], device=DEVICE)
    seq = torch.searchsorted(s.cu[1:], n, right=True)
    return rows.reshape(s.S, s.Hq, s.max_q, -1)[seq, :, n - s.cu[seq]]


def _plain_append(s):
    n = torch.arange(s.k_new.shape[0], device=DEVICE)
    seq = torch.searchsorted(s.cu[1:], n, right=True)
    j = s.used[seq] - s.new[seq] + n - s.cu[seq]
    page, slot = s.table[seq, j // s.page].long(), j % s.page
    s.k[page, slot], s.v[page, slot] = s.k_new.to(s.k.dtype), s.v_new.to(s.v.dtype)
    s.weights[page, :, slot] = 0.0
    return [s.k, s.v, s.weights]


def _plain_attention(s):
    scores = _scores(s)
    top = scores.max(-1, keepdim=True).values
    p = torch.exp(scores - top)
    del scores
    total = p.sum(-1, keepdim=True)
    o = _packed(s, torch.matmul(p, _key_rows(s, s.v)) / total).to(s.q.dtype)
    return [o] if s.lse is None else [o, _packed(s, top + torch.log(total))[..., 0].t().contiguous()]


def _plain_weights(s):
    i = torch.arange(s.max_q, device=DEVICE)
    lse = s.lse.t()[(s.cu[:-1, None] + i).clamp(max=s.q.shape[0] - 1)].transpose(1, 2).reshape(s.S, s.Hkv, -1, s.max_q)
    p = torch.exp(_scores(s).view(s.S, s.Hkv, -1, s.max_q, s.max_k) - lse[..., None])
    p = p.masked_fill_((i >= s.new[:, None])[:, None, None, :, None], 0.0).sum((2, 3)).transpose(1, 2)          # [S, longest, Hkv]
    j = _all_keys(s)
    there = j < s.used[:, None]
    slots = _slots(s, s.table, j)[there]
    page, slot = slots // s.page, slots % s.page
    p = p[there]
    s.weights[page, :, slot] = p + s.before[page, :, slot] * s.decay if s.decay else p
    return [s.weights]


def _plain_evict(s):
    j = _all_keys(s)
    at = _slots(s, s.table, j)
    w = s.weights[at // s.page, :, at % s.page].transpose(1, 2)                                 # [S, Hkv, longest]
    used = s.used[:, None]
    stays = (j < s.first) | (j >= used - s.recent)
    w = w.masked_fill(stays[:, None], math.inf).masked_fill((j >= used)[:, None], -math.inf)
    order = torch.sort(w, dim=-1, descending=True, stable=True).indices[..., :s.keep]
    if order.shape[-1] < s.keep:
        order = torch.nn.functional.pad(order, (0, s.keep - order.shape[-1]), value=s.max_k)
    room = torch.arange(s.keep, device=DEVICE)
    to_used = s.used.clamp(max=s.keep)
    there = room < to_used[:, None]
    kept = torch.sort(order.masked_fill(~there[:, None], s.max_k), -1).values.masked_fill(~there[:, None], -1)
    # rows of every head from where it was to where it goes
    seq, head, place = torch.nonzero(there[:, None].expand_as(kept), as_tuple=True)
    key = kept[seq, head, place]
    page, slot = s.table[seq, key // s.page].long(), key % s.page
    to_page, to_slot = s.to_table[seq, place // s.page].long(), place % s.page
    s.to_k[to_page, to_slot, head], s.to_v[to_page, to_slot, head] = s.k[page, slot, head], s.v[page, slot, head]
    s.to_weights[to_page, head, to_slot] = s.weights[page, head, slot]
    return [s.to_k, s.to_v, s.to_weights, kept.to(torch.int32), to_used]


# ---- the package's operators ---------------------------------------------------------------------------------------------------
def _own(s):
    import paper_2502_04507_amd as sta
    if s.kind == "append":
        sta.sta_paged_append(s.k_new, s.v_new, s.cu, s.cache, s.max_q, weights=s.weights)
        return [s.k, s.v, s.weights]
    if s.kind == "attention":
        sta.sta_paged_forward(s.q, s.o, s.cu, s.cache, s.max_q, s.max_k, causal=s.causal, lse=s.lse, workspace=s.workspace)
        return [s.o] if s.lse is None else [s.o, s.lse]
    if s.kind == "weights":
        sta.sta_paged_weights(s.q, s.lse, s.weights, s.cu, s.cache, s.max_q, s.max_k, before=s.before, decay=s.decay)
        return [s.weights]
    sta.sta_paged_evict(s.cache, s.weights, s.into, s.to_weights, s.kept, first=s.first, recent=s.recent)
    return [s.to_k, s.to_v, s.to_weights, s.kept, s.to_used]


def run(s):
    if own:
        return _own(s)
    if s.kind == "append":
        return _plain_append(s)
    if s.kind == "attention":
        return _plain_attention(s)
    return _plain_weights(s) if s.kind == "weights" else _plain_evict(s)


# ---- the definitions in 64 bits ------------------------------------------------------------------------------------------------
def exact(case, seed):
    s = prepare(case, seed)
    table, used = s.table.tolist(), s.used.tolist()

    def places(row, n):
        """Pages and slots of a sequence's first n keys."""
        return (torch.tensor([row[j // s.page] for j in range(n)], dtype=torch.long, device=DEVICE),
                torch.tensor([j % s.page for j in range(n)], dtype=torch.long, device=DEVICE))

    if case["kind"] == "evict":
        to_k, to_v = torch.zeros(s.to_k.shape, dtype=torch.float64, device=DEVICE), torch.zeros(s.to_v.shape, dtype=torch.float64, device=DEVICE)
        to_w, kept = torch.zeros(s.to_weights.shape, dtype=torch.float64, device=DEVICE), torch.full_like(s.kept, -1)
        for n, (row, to_row, lk) in enumerate(zip(table, s.to_table.tolist(), used)):
            page, slot = places(row, lk)
            to_page, to_slot = places(to_row, min(lk, s.keep))
            for h in range(s.Hkv):
                w = s.weights[page, h, slot].double()
                key = torch.arange(lk, device=DEVICE)
                if lk > s.keep:
                    middle = slice(s.first, lk - s.recent)
                    # the least go first, and of equal ones the last
                    least = torch.sort(w[middle].flip(0), stable=True).indices[:lk - s.keep]
                    gone = lk - s.recent - 1 - least
                    stay = torch.ones(lk, dtype=torch.bool, device=DEVICE)
                    stay[gone] = False
                    key = key[stay]
                kept[n, h, :len(key)] = key.int()
                to_k[to_page, to_slot, h] = s.k[page[key], slot[key], h].double()
                to_v[to_page, to_slot, h] = s.v[page[key], slot[key], h].double()
                to_w[to_page, h, to_slot] = w[key]
        return [to_k, to_v, to_w, kept, torch.tensor([min(x, s.keep) for x in used], dtype=torch.int32, device=DEVICE)]

    new, cu = _lengths(case["new"]), s.cu.tolist()
    if case["kind"] == "append":
        k, v, weights = s.k.double(), s.v.double(), s.weights.double()
        for n, (row, lq, lk) in enumerate(zip(table, new, used)):
            page, slot = (x[lk - lq:] for x in places(row, lk))
            k[page, slot], v[page, slot] = s.k_new[cu[n]:cu[n + 1]].double(), s.v_new[cu[n]:cu[n + 1]].double()
            weights[page, :, slot] = 0.0
        return [k, v, weights]

    group = s.Hq // s.Hkv
    o, lse = torch.zeros(s.q.shape, dtype=torch.float64, device=DEVICE), torch.zeros((s.Hq, s.q.shape[0]), dtype=torch.float64, device=DEVICE)
    weights = torch.zeros((s.k.shape[0], s.Hkv, s.page), dtype=torch.float64, device=DEVICE)
    for n, (row, lq, lk) in enumerate(zip(table, new, used)):
        page, slot = places(row, lk)
        rows = slice(cu[n], cu[n] + lq)
        for h in range(s.Hq):
            scores = s.q[rows, h].double() @ s.k[page, slot, h // group].double().T / math.sqrt(s.D)
            if s.causal:
                scores += torch.full_like(scores, -math.inf).triu(lk - lq + 1)
            if case["kind"] == "weights":
                if h % group == 0:
                    weights[page, h // group, slot] = s.before[page, h // group, slot].double() * s.decay if s.decay else 0.0
                weights[page, h // group, slot] += torch.exp(scores - s.lse[h, rows, None].double()).sum(0)
                continue
            z = torch.logsumexp(scores, -1)
            o[rows, h], lse[h, rows] = torch.exp(scores - z[:, None]) @ s.v[page, slot, h // group].double(), z
    if case["kind"] == "weights":
        return [weights]
    return [o, lse] if case["lse"] else [o]


def _seen(lq, lk, causal):
    """Pairs of a row and a key that it sees."""
    return lq * (lk - lq) + lq * (lq + 1) // 2 if causal else lq * lk


def work(case):
    Hkv, D, used = case["Hkv"], case["D"], _lengths(case["used"])
    if case["kind"] == "evict":
        stay = sum(min(x, case["keep"]) for x in used)
        # every weight, the rows that stay out and in, their weights and indices
        return {"bytes": 4 * Hkv * sum(used) + Hkv * stay * (2 * 2 * D * 2 + 4 + 4), "flops": float(Hkv * sum(used))}
    new = _lengths(case["new"])
    if case["kind"] == "append":
        return {"bytes": sum(new) * Hkv * (2 * D * ((4 if case["f32"] else 2) + 2) + 4), "flops": float(sum(new) * Hkv * 2 * D)}
    Hq, rows = case["Hq"], 2 * D * case["Hq"] * sum(new)
    pairs = sum(_seen(a, b, case.get("causal", True)) for a, b in zip(new, used))
    if case["kind"] == "weights":
        return {"bytes": rows + 4 * Hq * sum(new) + Hkv * sum(used) * (2 * D + (8 if case["decay"] else 4)), "flops": 2.0 * D * Hq * pairs}
    return {"bytes": 2 * rows + (4 * Hq * sum(new) if case["lse"] else 0) + Hkv * sum(used) * 2 * 2 * D, "flops": 4.0 * D * Hq * pairs}
