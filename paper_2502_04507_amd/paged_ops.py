"""Binding of the operators on a cache of keys and values in pages.  Same names as the C entry points of libsta.so; tensors are torch tensors used as
device-memory handles, outputs are given by the caller, the stream is torch's current HIP stream unless one is given.
"""
import ctypes

import torch

from .binding import STA_BF16, STA_F32, _check, _dev, _fast, _stream_ptr, load_library
from .layer_ops import _HeadRows, _bounds, _int32, _lse_ptr, _packed_counts, _packed_rows


class _PagedCache(ctypes.Structure):
    _fields_ = [("k", _HeadRows), ("v", _HeadRows), ("pages", ctypes.c_int64), ("page_size", ctypes.c_int), ("table", ctypes.c_void_p),
                ("table_row", ctypes.c_int64), ("table_pages", ctypes.c_int), ("used", ctypes.c_void_p),
                ("numbers_by_sequence", ctypes.c_int)]


def _bind(lib):
    """Argument types of this module's entry points."""
    if getattr(lib, "_paged_ops_bound", False):
        return lib
    vp, ci, cf, sz, i64 = ctypes.c_void_p, ctypes.c_int, ctypes.c_float, ctypes.c_size_t, ctypes.c_int64
    rows, cache = ctypes.POINTER(_HeadRows), ctypes.POINTER(_PagedCache)
    lib.sta_paged_append.argtypes = [rows, rows, i64, vp, cache, ci, ci, ci, vp, vp]
    lib.sta_paged_workspace_bytes.argtypes = [ci, ci, ci, ci, i64, ci, ci]
    lib.sta_paged_workspace_bytes.restype = sz
    lib.sta_paged_forward.argtypes = [rows, rows, vp, i64, vp, cache, ci, ci, ci, ci, ci, cf, vp, sz, vp]
    lib.sta_paged_weights.argtypes = [rows, vp, i64, vp, cache, ci, ci, ci, ci, ci, cf, vp, cf, vp, vp]
    lib.sta_paged_evict.argtypes = [cache, vp, cache, vp, vp, ci, ci, ci, ci, ci, vp]
    lib._paged_ops_bound = True
    return lib


def _lib():
    return _bind(load_library())


class StaPagedCache:
    """A cache in pages: k, v (device bf16 [pages, page_size, Hkv, D], laid out alike, channels adjacent; strided views such as halves of one tensor or of
    [pages, Hkv, page_size, D] turned around), table (device int32 [S, n]: the pages of every sequence in the order of its keys), used (device int32 [S]: how many
    keys it has, at most `room`).  shared: the numbers of the keys (gathered weights, float32 of weights_shape) are every sequence's own, [S, Hkv, room], in place of [pages, Hkv, page_size],
    beside the rows; pages that stand in the rows of several sequences need that, where numbers are gathered at all.  The tensors are kept and used as they are: what they hold may change from
    call to call, other tensors need another cache."""

    def __init__(self, k, v, table, used, shared=False):
        if k.dim() != 4 or k.shape != v.shape or k.dtype != torch.bfloat16 or v.dtype != torch.bfloat16:
            raise ValueError("k and v must be bfloat16 [pages, page_size, Hkv, D]")
        if k.stride() != v.stride():
            raise ValueError("k and v must be laid out alike")
        if table.dtype != torch.int32 or table.dim() != 2 or (table.shape[1] > 1 and table.stride(1) != 1):
            raise ValueError("table must be int32 [S, n], a row's entries adjacent")
        if used.dtype != torch.int32 or used.shape != table.shape[:1]:
            raise ValueError("used must be int32 [S]")
        if not (k.is_cuda and v.is_cuda and table.is_cuda):
            raise ValueError("a cache must live in device memory")
        self._tensors = k, v, table, used
        self.pages, self.page_size, self.Hkv, self.D = k.shape
        self.S = _int32(table.shape[0], "the number of sequences")
        page, token, head, channel = k.stride()
        if channel != 1:
            raise ValueError("the channels of k and v must be adjacent")
        heads = _int32(self.Hkv, "the number of heads")
        # a tensor without elements has no address; nothing of it is touched
        self._c = _PagedCache(_HeadRows(k.data_ptr() or 16, page, token, head, heads, STA_BF16), _HeadRows(v.data_ptr() or 16, page, token, head, heads, STA_BF16),
                              self.pages, _int32(self.page_size, "the page size"), table.data_ptr() or 16, table.stride(0), _int32(table.shape[1], "the pages of a row"),
                              _dev(used, "used") or 16, int(bool(shared)))
        # for the extension: where the struct is, and what goes with it
        outer, _, inner = self.weights_shape
        self._at = (ctypes.addressof(self._c), self.S, heads, self.D, outer, inner)

    # Read only: calls take the addresses that were looked up above.
    k = property(lambda self: self._tensors[0])
    v = property(lambda self: self._tensors[1])
    table = property(lambda self: self._tensors[2])
    used = property(lambda self: self._tensors[3])

    @property
    def room(self):
        """Keys that a sequence can have."""
        return self.table.shape[1] * self.page_size

    @property
    def shared(self):
        return bool(self._c.numbers_by_sequence)

    @property
    def weights_shape(self):
        """Of the keys' numbers."""
        return (self.S, self.Hkv, self.room) if self.shared else (self.pages, self.Hkv, self.page_size)


def _weights_ptr(w, cache, name):
    """Numbers of the keys."""
    if w is None:
        return None
    if w.dtype != torch.float32 or w.shape != cache.weights_shape:
        raise ValueError("%s must be float32 [%s]" % (name, "S, Hkv, room" if cache.shared else "pages, Hkv, page_size"))
    return _dev(w, name) or 16


def sta_paged_append(k, v, cu, cache, max_new, weights=None, stream=None):
    """New rows k, v (bf16 or float32 [tokens, Hkv, D], strided views with adjacent channels) into their pages: cu int32 [S + 1] where the sequences' tokens
    begin; cache.used counts them already; weights: the keys' numbers, set to 0 for the new keys, or None; max_new: upper bound of a sequence's tokens."""
    if stream is None:
        status = _fast().paged_append(k, v, cu, cache._at, max_new, weights)
        if status is not None:
            _check(status)
            return cache
    rows = []
    for t, name in ((k, "k"), (v, "v")):
        if t.dim() != 3 or t.shape != (k.shape[0], cache.Hkv, cache.D):
            raise ValueError("%s must be [tokens, Hkv, D]" % name)
        if t.dtype not in (torch.bfloat16, torch.float32):
            raise TypeError("%s must be bfloat16 or float32" % name)
        if not t.is_cuda:
            raise ValueError("%s must live in device memory" % name)
        token, head, channel = t.stride()
        if channel != 1:
            raise ValueError("the channels of %s must be adjacent" % name)
        rows.append(_HeadRows(t.data_ptr() or 16, 0, token, head, cache._c.k.heads, STA_F32 if t.dtype == torch.float32 else STA_BF16))
    _check(_lib().sta_paged_append(rows[0], rows[1], k.shape[0], _bounds(cu, "cu", cache.S + 1), cache._c, cache.S, _int32(max_new, "max_new"), cache.D,
                                   _weights_ptr(weights, cache, "weights"), _stream_ptr(stream)))
    return cache


def sta_paged_workspace_bytes(Hq, Hkv, D, S, tokens_q, max_q, max_k) -> int:
    sizes = [_int32(x, name) for x, name in ((Hq, "Hq"), (Hkv, "Hkv"), (D, "D"), (S, "S"))]
    return int(_lib().sta_paged_workspace_bytes(*sizes, int(tokens_q), _int32(max_q, "max_q"), _int32(max_k, "max_k")))


def _paged_queries(q, cu_q, cache, max_q, max_k):
    """Tokens and query heads, and the two bounds."""
    if q.dim() != 3:
        raise ValueError("expect [tokens, heads, D] tensors")
    S, max_q, max_k = _packed_counts(cu_q, max_q, max_k)
    if S != cache.S:
        raise ValueError("cu_q must have an entry more than the cache has sequences")
    return q.shape[0], _int32(q.shape[1], "the number of heads"), max_q, max_k


def sta_paged_forward(q, o, cu_q, cache, max_q, max_k, causal=True, scale=0.0, lse=None, workspace=None, stream=None):
    """sta_packed_forward against a cache in pages: q, o bf16 [tokens, Hq, D], cu_q int32 [S + 1]; lse float32 [Hq, tokens] or None; max_q, max_k upper bounds of
    the sequences' tokens and keys; workspace: device bytes, at least sta_paged_workspace_bytes(...), or None."""
    if stream is None:
        status = _fast().paged_forward(q, o, cu_q, cache._at, max_q, max_k, causal, scale, lse, workspace)
        if status is not None:
            _check(status)
            return o
    tq, Hq, max_q, max_k = _paged_queries(q, cu_q, cache, max_q, max_k)
    ws, nbytes = (None, 0) if workspace is None else (_dev(workspace, "workspace"), workspace.numel() * workspace.element_size())
    _check(_lib().sta_paged_forward(_packed_rows(q, "q", tq, Hq, cache.D), _packed_rows(o, "o", tq, Hq, cache.D), _lse_ptr(lse, Hq, tq), tq,
                                    _bounds(cu_q, "cu_q", cache.S + 1), cache._c, cache.S, max_q, max_k, cache.D, int(bool(causal)), scale, ws, nbytes,
                                    _stream_ptr(stream)))
    return o


def sta_paged_weights(q, lse, weights, cu_q, cache, max_q, max_k, before=None, decay=1.0, causal=True, scale=0.0, stream=None):
    """What every key of the cache gathers from these rows, added to decay times before (None: nothing; may be weights): weights float32 of
    cache.weights_shape (of pages that several sequences have, the numbers of a shared cache alone mean something); q bf16 [tokens, Hq, D] and lse float32 [Hq, tokens] as
    sta_paged_forward had and wrote them."""
    if stream is None:
        status = _fast().paged_weights(q, lse, weights, cu_q, cache._at, max_q, max_k, before, decay, causal, scale)
        if status is not None:
            _check(status)
            return weights
    tq, Hq, max_q, max_k = _paged_queries(q, cu_q, cache, max_q, max_k)
    if lse is None or weights is None:
        raise ValueError("lse and weights are needed")
    _check(_lib().sta_paged_weights(_packed_rows(q, "q", tq, Hq, cache.D), _lse_ptr(lse, Hq, tq), tq, _bounds(cu_q, "cu_q", cache.S + 1), cache._c, cache.S, max_q,
                                    max_k, cache.D, int(bool(causal)), scale, _weights_ptr(before, cache, "before"), decay,
                                    _weights_ptr(weights, cache, "weights"), _stream_ptr(stream)))
    return weights


def sta_paged_evict(cache, weights, into, into_weights, kept, first=0, recent=0, stream=None):
    """Keeps of every sequence and key head kept.shape[2] keys: the first and recent ones, and of the others those of the greatest weights.  Their rows go to the pages of
    into, another StaPagedCache whose used is written; their weights, of cache.weights_shape, to into_weights, of into.weights_shape (or None); kept int32
    [S, Hkv, keep]: which they were, -1 where there are fewer."""
    if stream is None:
        status = _fast().paged_evict(cache._at, weights, into._at, into_weights, kept, first, recent)
        if status is not None:
            _check(status)
            return into
    if into.S != cache.S or into.Hkv != cache.Hkv or into.D != cache.D:
        raise ValueError("both caches must have the same sequences, heads and channels")
    if kept.dtype != torch.int32 or kept.dim() != 3 or kept.shape[:2] != (cache.S, cache.Hkv):
        raise ValueError("kept must be int32 [S, Hkv, keep]")
    if weights is None:
        raise ValueError("weights are needed")
    _check(_lib().sta_paged_evict(cache._c, _weights_ptr(weights, cache, "weights"), into._c, _weights_ptr(into_weights, into, "into_weights"),
                                  _dev(kept, "kept") or 16, cache.S, _int32(kept.shape[2], "keep"), _int32(first, "first"), _int32(recent, "recent"), cache.D,
                                  _stream_ptr(stream)))
    return into
