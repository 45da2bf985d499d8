"""Binding of the operators around the attention: norms and rotary positions of query and key rows, attention over packed
sequences.  Same names as the C entry points of libsta.so; tensors are torch tensors used as device-memory handles, outputs are
given by the caller, the stream is torch's current HIP stream unless one is given.
"""
import ctypes
import operator

import torch

from .binding import STA_BF16, STA_F32, StaError, _check, _dev, _fast, _i3, _stream_ptr, load_library, sta_strerror  # noqa: F401

STA_ROPE_NONE, STA_ROPE_LINEAR, STA_ROPE_NTK, STA_ROPE_YARN = 0, 1, 2, 3
_DTYPES = {torch.bfloat16: STA_BF16, torch.float32: STA_F32}


def _int32(x, name):
    """x as the library's int: ctypes would drop the upper bits."""
    x = int(x)
    if not -2 ** 31 <= x < 2 ** 31:
        raise ValueError("%s does not fit 32 bits" % name)
    return x


class _HeadRows(ctypes.Structure):
    _fields_ = [("data", ctypes.c_void_p), ("batch", ctypes.c_int64), ("token", ctypes.c_int64), ("head", ctypes.c_int64),
                ("heads", ctypes.c_int), ("dtype", ctypes.c_int)]


class _Rotary(ctypes.Structure):
    _fields_ = [("steps", ctypes.c_void_p), ("positions", ctypes.c_void_p), ("position_batch", ctypes.c_int64),
                ("position_token", ctypes.c_int64), ("channels", ctypes.c_int), ("pairs", ctypes.c_int * 3),
                ("interleaved", ctypes.c_int), ("magnitude", ctypes.c_float)]


def _bind(lib):
    """Argument types of this module's entry points."""
    if getattr(lib, "_layer_ops_bound", False):
        return lib
    vp, ci, cf, sz, rows, i3 = (ctypes.c_void_p, ctypes.c_int, ctypes.c_float, ctypes.c_size_t, ctypes.POINTER(_HeadRows),
                                ctypes.c_void_p)
    lib.sta_rope_steps.argtypes = [ci, ctypes.c_double, ci, ctypes.c_double, ctypes.c_double, vp, ctypes.POINTER(cf)]
    lib.sta_rope.argtypes = [rows, rows, ci, ci, ci, ci, ctypes.POINTER(_Rotary), ci, vp]
    lib.sta_qk_norm_rope.argtypes = [rows] * 6 + [vp, vp, ci, cf, ctypes.POINTER(_Rotary), ci, ci, ci, i3, i3, vp]
    lib.sta_qk_norm_rope_workspace_bytes.argtypes = [ci]
    lib.sta_qk_norm_rope_workspace_bytes.restype = sz
    lib.sta_qk_norm_rope_backward.argtypes = [rows] * 8 + [vp, vp, ci, vp, vp, cf, ctypes.POINTER(_Rotary), ci, ci, ci, i3, i3, vp, sz, vp]
    i64 = ctypes.c_int64
    lib.sta_packed_workspace_bytes.argtypes = [ci, ci, ci, ci, i64, ci, ci]
    lib.sta_packed_workspace_bytes.restype = sz
    lib.sta_packed_forward.argtypes = [rows] * 4 + [vp, i64, i64, vp, vp, vp, ci, ci, ci, ci, ci, cf, vp, sz, vp]
    lib.sta_packed_backward_workspace_bytes.argtypes = [ci, i64]
    lib.sta_packed_backward_workspace_bytes.restype = sz
    lib.sta_packed_backward.argtypes = [rows] * 5 + [vp] + [rows] * 3 + [i64, i64, vp, vp, ci, ci, ci, ci, ci, cf, vp, sz, vp]
    lib._layer_ops_bound = True
    return lib


def _lib():
    return _bind(load_library())


class StaRotary:
    """Rotary positions: steps (device int64 [channels / 2], turns per position in units of 2^-64, see sta_rope_steps), positions (device
    int32: [N] or [B, N] on one axis, [N, 3] or [B, N, 3] on three; None: the places in a grid, or 0 .. N - 1), pairs (rotated pairs of
    every axis; default: all on the first), interleaved (neighbouring channels form a pair, not halves), magnitude (factor on what is
    rotated)."""

    def __init__(self, steps, positions=None, pairs=None, interleaved=False, magnitude=1.0):
        if steps.dtype != torch.int64 or steps.dim() != 1:
            raise ValueError("steps must be int64 [channels / 2]")
        pairs = [_int32(n, "pairs") for n in ((steps.numel(),) if pairs is None else pairs)]
        if not 1 <= len(pairs) <= 3 or min(pairs) < 0 or sum(pairs) != steps.numel():
            raise ValueError("pairs must have one to three entries that sum to the number of steps")
        axes = 3 if any(pairs[1:]) else 1
        pairs += [0] * (3 - len(pairs))
        self.steps, self.positions, self.interleaved, self.magnitude = steps, positions, bool(interleaved), float(magnitude)
        if not self.magnitude > 0.0:
            raise ValueError("magnitude must be positive")
        ptr, self._B, self._N, batch, token = None, None, None, 0, 0
        if positions is not None:
            if positions.dtype != torch.int32:
                raise ValueError("positions must be int32")
            shape, stride = tuple(positions.shape), positions.stride()
            if axes == 3:
                if len(shape) not in (2, 3) or shape[-1] != 3 or stride[-1] != 1:
                    raise ValueError("positions on three axes must be [N, 3] or [B, N, 3], the three adjacent")
                shape, stride = shape[:-1], stride[:-1]
            elif len(shape) not in (1, 2):
                raise ValueError("positions on one axis must be [N] or [B, N]")
            if len(shape) == 2:
                self._B, batch = shape[0], stride[0]
            self._N, token = shape[-1], stride[-1]
            if not positions.is_cuda:
                raise ValueError("positions must live in device memory")
            ptr = positions.data_ptr()
        self.channels = 2 * steps.numel()
        self._c = _Rotary(_dev(steps, "steps"), ptr, batch, token, self.channels, (ctypes.c_int * 3)(*pairs), int(self.interleaved),
                          self.magnitude)
        # for the extension: where the struct is, and which tokens the positions are for
        self._at = (ctypes.addressof(self._c), -1 if self._N is None else self._N, -1 if self._B is None else self._B)

    def _struct(self, B, N):
        if self._N is not None and (self._N != N or self._B not in (None, B)):
            raise ValueError("positions do not match the tokens")
        return self._c


def sta_rope_steps(channels, theta=10000.0, scaling=STA_ROPE_NONE, factor=1.0, original_positions=4096):
    """Turns per position of every pair in units of 2^-64 (host int64 tensor [channels / 2]) and the magnitude."""
    channels = _int32(channels, "channels")
    if channels < 2:
        _check(2)
    steps, magnitude = torch.empty(channels // 2, dtype=torch.int64), ctypes.c_float(1.0)
    _check(_lib().sta_rope_steps(channels, float(theta), _int32(scaling, "scaling"), float(factor), float(original_positions), steps.data_ptr(),
                                 ctypes.byref(magnitude)))
    return steps, float(magnitude.value)


def _sizes(t):
    """B, N and D of the first [B, N, H, D] tensor."""
    B, N, _, D = t.shape
    return _int32(B, "the batch"), _int32(N, "the number of tokens"), _int32(D, "the number of channels")


def _rows(t, name, B, N, D):
    """One [B, N, H, D] tensor, its channels adjacent."""
    shape = t.shape
    _int32(shape[2] if len(shape) == 4 else 0, "the number of heads")
    if len(shape) != 4 or shape[0] != B or shape[1] != N or shape[3] != D:
        raise ValueError("%s must be [B, N, H, D] like the others" % name)
    dtype = _DTYPES.get(t.dtype)
    if dtype is None:
        raise TypeError("only bfloat16 and float32 tensors are supported")
    if not t.is_cuda:
        raise ValueError("%s must live in device memory" % name)
    batch, token, head, channel = t.stride()
    if channel != 1 and D > 1:
        raise ValueError("the channels of %s must be adjacent" % name)
    # a tensor without elements has no address; nothing of it is touched
    return _HeadRows(t.data_ptr() or 16, batch, token, head, shape[2], dtype)


def sta_rope(xs, outs, rotary, inverse=False, stream=None):
    """Rotation of one to three [B, N, H, D] tensors (or strided views with adjacent channels) into outs, which may be the tensors
    themselves; inverse: back, which is the gradient."""
    if stream is None:
        status = _fast().rope(xs, outs, rotary._at, inverse)
        if status is not None:
            _check(status)
            return outs
    xs, outs = ([xs], [outs]) if isinstance(xs, torch.Tensor) else (list(xs), list(outs))
    n = len(xs)
    if not 1 <= n <= 3 or len(outs) != n:
        raise ValueError("expect one to three tensors and as many outputs")
    if xs[0].dim() != 4:
        raise ValueError("expect [B, N, H, D] tensors")
    B, N, D = _sizes(xs[0])
    a = (_HeadRows * n)(*[_rows(t, "input", B, N, D) for t in xs])
    b = (_HeadRows * n)(*[_rows(t, "output", B, N, D) for t in outs])
    _check(_lib().sta_rope(a, b, n, B, N, D, rotary._struct(B, N), int(bool(inverse)), _stream_ptr(stream)))
    return outs


def _weights(ws, D):
    """Addresses of the two weights and their type."""
    dtype = None
    ptrs = []
    for w in ws:
        if w is None:
            ptrs.append(None)
            continue
        if w.shape != (D,) or w.dtype not in _DTYPES or (dtype is not None and _DTYPES[w.dtype] != dtype):
            raise ValueError("weights must be [D] of one type, bfloat16 or float32")
        dtype = _DTYPES[w.dtype]
        ptrs.append(_dev(w, "weight"))
    return ptrs, STA_F32 if dtype is None else dtype


def _grid_tile(grid, tile):
    if tile is not None and grid is None:
        raise ValueError("a tile needs a grid")
    return None if grid is None else _i3(grid), None if tile is None else _i3(tile)


def sta_qk_norm_rope(q, k, v, q_out, k_out, v_out, q_weight, k_weight, rotary, eps=1e-6, grid=None, tile=None, stream=None):
    """RMS norm with weight [D] (None: ones) and rotation (rotary None: none) of query and key rows; v (may be None) is moved along.  All
    tensors [B, N, H, D], strided views with adjacent channels.  With grid and tile the tokens go from raster to tiled order; a [B, H, N, D]
    tensor for sta_forward is given as out.transpose(1, 2)."""
    if stream is None:
        status = _fast().norm_rope(q, k, v, q_out, k_out, v_out, q_weight, k_weight, None if rotary is None else rotary._at, eps, grid, tile)
        if status is not None:
            _check(status)
            return q_out, k_out, v_out
    if q.dim() != 4:
        raise ValueError("expect [B, N, H, D] tensors")
    if (v is None) != (v_out is None):
        raise ValueError("v and v_out go together")
    B, N, D = _sizes(q)
    rows = [None if t is None else _rows(t, name, B, N, D) for t, name in ((q, "q"), (k, "k"), (v, "v"), (q_out, "q_out"), (k_out, "k_out"), (v_out, "v_out"))]
    (wq, wk), dtype = _weights((q_weight, k_weight), D)
    g, t = _grid_tile(grid, tile)
    _check(_lib().sta_qk_norm_rope(*rows, wq, wk, dtype, eps, None if rotary is None else rotary._struct(B, N), B, N, D, g, t,
                                   _stream_ptr(stream)))
    return q_out, k_out, v_out


def sta_qk_norm_rope_workspace_bytes(D) -> int:
    return int(_lib().sta_qk_norm_rope_workspace_bytes(_int32(D, "D")))


def sta_qk_norm_rope_backward(q, k, d_q_out, d_k_out, d_v_out, d_q, d_k, d_v, q_weight, k_weight, d_q_weight, d_k_weight, rotary, workspace,
                              eps=1e-6, grid=None, tile=None, stream=None):
    """Gradients of sta_qk_norm_rope: d_*_out laid out like its outputs, d_q, d_k, d_v like its inputs; d_q_weight, d_k_weight float32 [D] or None;
    workspace: device bytes, at least sta_qk_norm_rope_workspace_bytes(D)."""
    if stream is None:
        status = _fast().norm_rope_backward(q, k, d_q_out, d_k_out, d_v_out, d_q, d_k, d_v, q_weight, k_weight, d_q_weight, d_k_weight,
                                            None if rotary is None else rotary._at, workspace, eps, grid, tile)
        if status is not None:
            _check(status)
            return d_q, d_k, d_v
    if q.dim() != 4:
        raise ValueError("expect [B, N, H, D] tensors")
    if (d_v is None) != (d_v_out is None):
        raise ValueError("d_v and d_v_out go together")
    B, N, D = _sizes(q)
    rows = [None if t is None else _rows(t, name, B, N, D) for t, name in
            ((q, "q"), (k, "k"), (d_q_out, "d_q_out"), (d_k_out, "d_k_out"), (d_v_out, "d_v_out"), (d_q, "d_q"), (d_k, "d_k"), (d_v, "d_v"))]
    (wq, wk), dtype = _weights((q_weight, k_weight), D)
    for w in (d_q_weight, d_k_weight):
        if w is not None and (w.shape != (D,) or w.dtype != torch.float32):
            raise ValueError("weight gradients must be float32 [D]")
    dw = [None if w is None else _dev(w, "weight gradient") for w in (d_q_weight, d_k_weight)]
    g, t = _grid_tile(grid, tile)
    ws, nbytes = (None, 0) if workspace is None else (_dev(workspace, "workspace"), workspace.numel() * workspace.element_size())
    _check(_lib().sta_qk_norm_rope_backward(*rows, wq, wk, dtype, *dw, eps, None if rotary is None else rotary._struct(B, N), B, N, D, g, t, ws,
                                            nbytes, _stream_ptr(stream)))
    return d_q, d_k, d_v


def _packed_rows(t, name, tokens, heads, D):
    """One [tokens, H, D] tensor, its channels adjacent."""
    if t.dim() != 3 or t.shape != (tokens, heads, D):
        raise ValueError("%s must be [tokens, heads, D] like the others" % name)
    if t.dtype != torch.bfloat16:
        raise TypeError("%s must be bfloat16" % name)
    if not t.is_cuda:
        raise ValueError("%s must live in device memory" % name)
    token, head, channel = t.stride()
    if channel != 1:
        raise ValueError("the channels of %s must be adjacent" % name)
    return _HeadRows(t.data_ptr() or 16, 0, token, head, heads, STA_BF16)


def _bounds(t, name, n):
    if t is None:
        return None
    if t.dtype != torch.int32 or t.shape != (n,):
        raise ValueError("%s must be int32 [%d]" % (name, n))
    return _dev(t, name)


def _packed_shapes(q, k):
    if q.dim() != 3 or k.dim() != 3:
        raise ValueError("expect [tokens, heads, D] tensors")
    (tq, Hq, D), (tk, Hkv, _) = q.shape, k.shape
    return tq, _int32(Hq, "the number of heads"), _int32(D, "the number of channels"), tk, _int32(Hkv, "the number of heads")


def _packed_counts(cu_q, max_q, max_k):
    S = _int32(cu_q.numel() - 1, "the number of sequences")
    if S < 0:
        raise ValueError("cu_q needs an entry more than there are sequences")
    return S, _int32(operator.index(max_q), "max_q"), _int32(operator.index(max_k), "max_k")


def _lse_ptr(lse, Hq, tq):
    if lse is None:
        return None
    if lse.dtype != torch.float32 or lse.shape != (Hq, tq):
        raise ValueError("lse must be float32 [Hq, tokens]")
    return _dev(lse, "lse") or 16


def sta_packed_workspace_bytes(Hq, Hkv, D, S, tokens_q, max_q, max_k) -> int:
    sizes = [_int32(x, name) for x, name in ((Hq, "Hq"), (Hkv, "Hkv"), (D, "D"), (S, "S"))]
    return int(_lib().sta_packed_workspace_bytes(*sizes, int(tokens_q), _int32(max_q, "max_q"), _int32(max_k, "max_k")))


def sta_packed_forward(q, k, v, o, cu_q, cu_k, max_q, max_k, causal=True, scale=0.0, lse=None, k_used=None, workspace=None, stream=None):
    """Attention over packed sequences: q, o bf16 [tokens, Hq, D], k, v bf16 [key tokens, Hkv, D] (strided views with adjacent channels); cu_q, cu_k
    int32 [S + 1] where the sequences begin, k_used int32 [S] or None; lse float32 [Hq, tokens] or None; max_q, max_k upper bounds of the lengths."""
    if stream is None:
        status = _fast().packed_forward(q, k, v, o, cu_q, cu_k, max_q, max_k, causal, scale, lse, k_used, workspace)
        if status is not None:
            _check(status)
            return o
    tq, Hq, D, tk, Hkv = _packed_shapes(q, k)
    S, max_q, max_k = _packed_counts(cu_q, max_q, max_k)
    ws, nbytes = (None, 0) if workspace is None else (_dev(workspace, "workspace"), workspace.numel() * workspace.element_size())
    _check(_lib().sta_packed_forward(_packed_rows(q, "q", tq, Hq, D), _packed_rows(k, "k", tk, Hkv, D), _packed_rows(v, "v", tk, Hkv, D),
                                     _packed_rows(o, "o", tq, Hq, D), _lse_ptr(lse, Hq, tq), tq, tk, _bounds(cu_q, "cu_q", S + 1),
                                     _bounds(cu_k, "cu_k", S + 1), _bounds(k_used, "k_used", S), S, max_q, max_k, D, int(bool(causal)), scale, ws,
                                     nbytes, _stream_ptr(stream)))
    return o


def sta_packed_backward_workspace_bytes(Hq, tokens_q) -> int:
    return int(_lib().sta_packed_backward_workspace_bytes(_int32(Hq, "Hq"), int(tokens_q)))


def sta_packed_backward(q, k, v, o, d_o, lse, d_q, d_k, d_v, cu_q, cu_k, max_q, max_k, workspace, causal=True, scale=0.0, stream=None):
    """Gradients of sta_packed_forward; tensors as there, workspace: device bytes, at least sta_packed_backward_workspace_bytes(Hq, tokens)."""
    if stream is None:
        status = _fast().packed_backward(q, k, v, o, d_o, lse, d_q, d_k, d_v, cu_q, cu_k, max_q, max_k, workspace, causal, scale)
        if status is not None:
            _check(status)
            return d_q, d_k, d_v
    tq, Hq, D, tk, Hkv = _packed_shapes(q, k)
    S, max_q, max_k = _packed_counts(cu_q, max_q, max_k)
    if lse is None:
        raise ValueError("lse is needed")
    _check(_lib().sta_packed_backward(_packed_rows(q, "q", tq, Hq, D), _packed_rows(k, "k", tk, Hkv, D), _packed_rows(v, "v", tk, Hkv, D),
                                      _packed_rows(o, "o", tq, Hq, D), _packed_rows(d_o, "d_o", tq, Hq, D), _lse_ptr(lse, Hq, tq),
                                      _packed_rows(d_q, "d_q", tq, Hq, D), _packed_rows(d_k, "d_k", tk, Hkv, D),
                                      _packed_rows(d_v, "d_v", tk, Hkv, D), tq, tk, _bounds(cu_q, "cu_q", S + 1), _bounds(cu_k, "cu_k", S + 1), S,
                                      max_q, max_k, D, int(bool(causal)), scale, _dev(workspace, "workspace"),
                                      workspace.numel() * workspace.element_size(), _stream_ptr(stream)))
    return d_q, d_k, d_v
