"""A kept scene: norms and rotation of queries and keys, a paged cache of keys and values, attention of a batch to a shared prefix.

The calls of include/httm.h that need no geometry of a merged layer.  A program that encodes a scene once and looks later images up in
it (or decodes tokens behind a common document) makes, per layer,

    q, k = rotary.norm_rotate(q, k, positions, ...)            # of the scene's own layers; in front of Httm.global_attention
    cache.append(batch, k, v, rotary=rotary, ...)               # new keys (normed and rotated on the way) and values into their pages
    out = cache.attention(batch, q)                             # softmax over the prefix and each sequence's own keys

with one CacheBatch for all layers of a step (it holds the sequences, their pages and the plan of the attention) and one KvCache per
layer.  Tensors are bf16 or fp16 CUDA tensors [heads][tokens][head_dim] with contiguous channels and any strides that are multiples
of 8 elements: views of a fused projection output [tokens][heads][head_dim] are fine.  Only marshalling happens here; every step runs
in the library's CUDA kernels, and there is no CPU fallback.
"""
from __future__ import annotations

import ctypes
import struct

import numpy as np
import torch

from . import binding
from .binding import ERR_INVALID_ARG, OK, HttmError, _Tensor

NORMS = {"none": 0, "rms": 1, "layer": 2}
_DTYPES = {torch.bfloat16: 0, torch.float16: 1}
_vp, _i32, _i64 = ctypes.c_void_p, ctypes.c_int32, ctypes.c_int64


class _RotaryConfig(ctypes.Structure):
    _fields_ = [(n, _i32) for n in ("device", "head_dim", "norm", "rotated_dim", "axes", "interleaved", "n_positions")] + [
        ("eps", ctypes.c_double), ("base", ctypes.c_double), ("frequencies", ctypes.POINTER(ctypes.c_double))]


_ROWS = struct.Struct("Pqq Pqq i4x PP".replace(" ", ""))               # httm_rows: x, y, heads, weight, bias
_ROWS_GRAD = struct.Struct("Pqq Pqq Pqq i4x PPP".replace(" ", ""))     # httm_rows_grad: x, dy, dx, heads, weight, dweight, dbias


class _BatchConfig(ctypes.Structure):
    _fields_ = [(n, _i32) for n in ("device", "heads", "kv_heads", "head_dim", "page_size", "causal")] + [("n_pages", _i64)]


class _Pages(ctypes.Structure):
    _fields_ = [("ptr", _vp), ("stride_page", _i64), ("stride_head", _i64), ("stride_slot", _i64)]


_lib = None


def _library():
    global _lib
    if _lib is None:
        L = binding.load_library()
        P = ctypes.POINTER
        L.httm_rotary_create.argtypes = [P(_RotaryConfig), P(_vp)]
        L.httm_rotary_destroy.argtypes = [_vp]
        L.httm_rotary_status.argtypes = [_vp, P(_i64)]
        L.httm_norm_rotate.argtypes = [_vp, _i32, _i64, _vp, _vp, _vp, _vp]
        L.httm_norm_rotate_backward.argtypes = [_vp, _i32, _i64, _vp, _vp, _vp, _vp]
        L.httm_batch_create.argtypes = [P(_BatchConfig), P(_vp)]
        L.httm_batch_destroy.argtypes = [_vp]
        L.httm_batch_status.argtypes = [_vp, P(_i64)]
        L.httm_batch_set.argtypes = [_vp, _i32, _vp, _vp, _vp, _i64, _vp, _i32, _vp]
        L.httm_cache_append.argtypes = [_vp, _i32, _Pages, _Pages, _Tensor, _Tensor, _vp, _vp, _vp, _vp, _vp]
        L.httm_cache_attention.argtypes = [_vp, _i32, _Pages, _Pages, _Tensor, _Tensor, ctypes.c_double, _vp]
        _lib = L
    return _lib


def _check(rc: int):
    if rc != OK:
        raise HttmError(rc, (_lib.httm_last_error(None) or b"").decode())


def _bad(message: str):
    raise HttmError(ERR_INVALID_ARG, message)


# The kernels of a call on a few tokens take 2 - 3 us, so what is done per call is kept small: attributes are asked for once, arguments are
# packed into a buffer that the handle keeps instead of into new structures, the current stream's address is asked for without building a
# stream object (norm_rotate on one token, from call to call: 13.0 -> 8.8 us; append of 64 tokens 9.4 -> 6.9).
_raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None)


def _stream(stream, device: int):
    if stream is not None:
        return stream.cuda_stream
    if _raw_stream is not None:
        return _raw_stream(device)
    return torch.cuda.current_stream(device).cuda_stream


def _rows(t: torch.Tensor, name: str, shape, dtype, device: int):
    """(address, stride of heads, stride of tokens)"""
    if t.dtype is not dtype or t.get_device() != device:
        _bad(f"{name}: expected a {dtype} tensor on cuda:{device}")
    if t.shape != shape:
        _bad(f"{name}: expected shape {tuple(shape)} [heads][tokens][head_dim]")
    sh, st, sc = t.stride()
    if sc != 1:
        _bad(f"{name}: channels must be contiguous")
    return t.data_ptr(), sh, st


def _vector(t, name: str, dim: int, device: int) -> int:
    if t is None:
        return 0
    if t.dtype is not torch.float32 or t.get_device() != device or t.shape != (dim,) or not t.is_contiguous():
        _bad(f"{name}: expected a contiguous float32 vector of head_dim = {dim} on cuda:{device}")
    return t.data_ptr()


def _kind(t: torch.Tensor, name: str) -> int:
    kind = _DTYPES.get(t.dtype)
    if kind is None:
        _bad(f"{name}: expected bfloat16 or float16")
    return kind


class _Handle:
    _destroy = ""

    def close(self):
        if getattr(self, "_h", None):
            getattr(self._lib, self._destroy)(self._h)
            self._h = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass

    def __enter__(self):
        return self

    def __exit__(self, *exc):
        self.close()

    def _handle(self):
        if not self._h:
            _bad("the handle is closed")
        return self._h


class Rotary(_Handle):
    """Norms of queries and keys for each head and their rotation by position (see httm_rotary_config in include/httm.h).

    axes = 2 rotates the first half of the rotated channels by the row and the second by the column of a patch; positions are then
    [tokens][2], else [tokens] or [tokens][1], int32.  norm: "layer", "rms" or "none".
    """

    _destroy = "httm_rotary_destroy"

    def __init__(self, head_dim: int, n_positions: int, axes: int = 1, rotated_dim: int = None, base: float = 10000.0, frequencies=None,
                 interleaved: bool = False, norm: str = "rms", eps: float = 1e-5, device: int = 0):
        self._lib = _library()
        if norm not in NORMS:
            _bad(f"norm must be one of {sorted(NORMS)}")
        rotated_dim = head_dim if rotated_dim is None else rotated_dim
        self.head_dim, self.axes, self.rotated_dim, self.norm, self.device = head_dim, axes, rotated_dim, norm, device
        f = None
        if frequencies is not None:
            f = np.ascontiguousarray(frequencies, dtype=np.float64)
            if axes < 1 or f.shape != (rotated_dim // axes // 2,):
                _bad("frequencies: expected rotated_dim / axes / 2 numbers")
            f = f.ctypes.data_as(ctypes.POINTER(ctypes.c_double))
        c = _RotaryConfig(device, head_dim, NORMS[norm], rotated_dim, axes, int(interleaved), n_positions, float(eps), float(base), f)
        h = _vp()
        _check(self._lib.httm_rotary_create(ctypes.byref(c), ctypes.byref(h)))
        self._h = h
        self._args = ctypes.create_string_buffer(2 * _ROWS_GRAD.size)   # the two row arguments of a call
        self._at = ctypes.addressof(self._args)

    def _positions(self, positions, tokens: int):
        if self.rotated_dim == 0:
            return None
        if positions is None:
            _bad("positions are missing")
        if positions.dtype is not torch.int32 or positions.get_device() != self.device or not positions.is_contiguous() or \
                (positions.shape != (tokens, self.axes) and (self.axes != 1 or positions.shape != (tokens,))):
            _bad(f"positions: expected a contiguous int32 tensor [{tokens}][{self.axes}] on cuda:{self.device}")
        return positions.data_ptr()

    @staticmethod
    def _first(q, k):
        first = q if q is not None else k
        if first is None:
            _bad("neither q nor k")
        if first.dim() != 3:
            _bad("expected [heads][tokens][head_dim]")
        return _kind(first, "q" if q is not None else "k"), first.shape[1], first.dtype

    def norm_rotate(self, q, k, positions, q_weight=None, k_weight=None, q_bias=None, k_bias=None, out_q=None, out_k=None, stream=None):
        """rotate(norm(x) * weight + bias) of q and of k (either may be None); returns (q', k'), in out_q / out_k where given (which may
        be q and k themselves)."""
        kind, tokens, dtype = self._first(q, k)
        dim, device = self.head_dim, self.device
        at, outs = [None, None], [None, None]
        if q is not None:
            shape = (q.shape[0], tokens, dim)
            x = _rows(q, "q", shape, dtype, device)
            if out_q is None:
                out_q = torch.empty(shape, dtype=dtype, device=q.device)
            _ROWS.pack_into(self._args, 0, *x, *_rows(out_q, "out_q", shape, dtype, device), shape[0], _vector(q_weight, "q_weight", dim, device),
                            _vector(q_bias, "q_bias", dim, device))
            at[0], outs[0] = self._at, out_q
        if k is not None:
            shape = (k.shape[0], tokens, dim)
            x = _rows(k, "k", shape, dtype, device)
            if out_k is None:
                out_k = torch.empty(shape, dtype=dtype, device=k.device)
            _ROWS.pack_into(self._args, _ROWS.size, *x, *_rows(out_k, "out_k", shape, dtype, device), shape[0],
                            _vector(k_weight, "k_weight", dim, device), _vector(k_bias, "k_bias", dim, device))
            at[1], outs[1] = self._at + _ROWS.size, out_k
        _check(self._lib.httm_norm_rotate(self._handle(), kind, tokens, self._positions(positions, tokens), at[0], at[1], _stream(stream, device)))
        return tuple(outs)

    def norm_rotate_backward(self, dq, dk, q, k, positions, q_weight=None, k_weight=None, q_bias=None, k_bias=None, out_q=None,
                             out_k=None, stream=None):
        """Gradients of norm_rotate from those of its outputs: (dq, dk, dq_weight, dq_bias, dk_weight, dk_bias), None for what was not given.
        out_q / out_k take the first two (and may be dq / dk or q / k themselves)."""
        kind, tokens, dtype = self._first(q, k)
        dim, device = self.head_dim, self.device
        at, outs, sums = [None, None], [None, None], [None] * 4
        for i, (x, dy, w, b, out, name) in enumerate(((q, dq, q_weight, q_bias, out_q, "q"), (k, dk, k_weight, k_bias, out_k, "k"))):
            if x is None:
                continue
            if dy is None:
                _bad(f"d{name} is missing")
            shape = (x.shape[0], tokens, dim)
            tx, tdy = _rows(x, name, shape, dtype, device), _rows(dy, "d" + name, shape, dtype, device)
            if out is None:
                out = torch.empty(shape, dtype=dtype, device=x.device)
            weight = _vector(w, name + "_weight", dim, device)
            _vector(b, name + "_bias", dim, device)
            to_w = to_b = 0
            if w is not None:
                sums[2 * i] = torch.empty(dim, dtype=torch.float32, device=x.device)
                to_w = sums[2 * i].data_ptr()
            if b is not None:
                sums[2 * i + 1] = torch.empty(dim, dtype=torch.float32, device=x.device)
                to_b = sums[2 * i + 1].data_ptr()
            _ROWS_GRAD.pack_into(self._args, i * _ROWS_GRAD.size, *tx, *tdy, *_rows(out, "out_" + name, shape, dtype, device), shape[0], weight, to_w, to_b)
            at[i], outs[i] = self._at + i * _ROWS_GRAD.size, out
        _check(self._lib.httm_norm_rotate_backward(self._handle(), kind, tokens, self._positions(positions, tokens), at[0], at[1],
                                                   _stream(stream, device)))
        return tuple(outs) + tuple(sums)

    def differentiable(self, q, k, positions, q_weight=None, k_weight=None, q_bias=None, k_bias=None):
        """norm_rotate with its gradient, for torch.autograd."""
        return _NormRotate.apply(self, q, k, positions, q_weight, k_weight, q_bias, k_bias)

    def status(self) -> int:
        """Waits for the device; raises if a position was outside the table."""
        v = _i64()
        _check(self._lib.httm_rotary_status(self._handle(), ctypes.byref(v)))
        return int(v.value)


class _NormRotate(torch.autograd.Function):
    @staticmethod
    def forward(ctx, rotary, q, k, positions, q_weight, k_weight, q_bias, k_bias):
        ctx.rotary = rotary
        ctx.save_for_backward(q, k, positions, q_weight, k_weight, q_bias, k_bias)
        return rotary.norm_rotate(q, k, positions, q_weight, k_weight, q_bias, k_bias)

    @staticmethod
    def backward(ctx, dq, dk):
        q, k, positions, q_weight, k_weight, q_bias, k_bias = ctx.saved_tensors

        def rows(dy):   # a gradient may come with any strides, broadcast channels among them
            if dy is None or (dy.stride(2) == 1 and dy.stride(0) % 8 == 0 and dy.stride(1) % 8 == 0 and dy.data_ptr() % 16 == 0):
                return dy
            return dy.contiguous()

        gq, gk, gqw, gqb, gkw, gkb = ctx.rotary.norm_rotate_backward(rows(dq), rows(dk), q, k, positions, q_weight, k_weight, q_bias, k_bias)
        return None, gq, gk, None, gqw, gkw, gqb, gkb


class CacheBatch(_Handle):
    """The sequences of one step over paged caches: see httm_batch_set in include/httm.h."""

    _destroy = "httm_batch_destroy"

    def __init__(self, heads: int, kv_heads: int, head_dim: int, page_size: int, n_pages: int, causal: bool = True, device: int = 0):
        self._lib = _library()
        self.heads, self.kv_heads, self.head_dim, self.page_size, self.n_pages, self.device = heads, kv_heads, head_dim, page_size, n_pages, device
        self.n_tokens = 0
        c = _BatchConfig(device, heads, kv_heads, head_dim, page_size, int(causal), n_pages)
        h = _vp()
        _check(self._lib.httm_batch_create(ctypes.byref(c), ctypes.byref(h)))
        self._h = h

    def set(self, tables, lengths, queries, prefix_pages=(), prefix_length: int = 0, stream=None):
        """tables: the pages of every sequence (a list of lists, or a 2-D integer array); lengths: its keys, the new ones included; queries:
        its query tokens; all on the host.  The plan is uploaded on `stream`."""
        self.n_tokens = 0
        n_seq = len(lengths)
        lengths, queries = (np.ascontiguousarray(x, dtype=np.int32) for x in (lengths, queries))
        if len(queries) != n_seq or len(tables) != n_seq or lengths.ndim != 1 or queries.ndim != 1:
            _bad("tables, lengths and queries: expected one entry per sequence")
        if isinstance(tables, np.ndarray):
            table = np.ascontiguousarray(tables, dtype=np.int32)
            if table.ndim != 2:
                _bad("tables: expected [sequences][pages]")
        else:
            table = np.full((n_seq, max((len(t) for t in tables), default=0)), -1, dtype=np.int32)
            for i, t in enumerate(tables):
                table[i, :len(t)] = t
        prefix = np.ascontiguousarray(prefix_pages, dtype=np.int32)
        if prefix.ndim != 1 or len(prefix) * self.page_size < prefix_length:
            _bad("prefix_pages: fewer pages than prefix_length takes")
        _check(self._lib.httm_batch_set(self._handle(), n_seq, lengths.ctypes.data, queries.ctypes.data, table.ctypes.data, table.shape[1],
                                        prefix.ctypes.data, int(prefix_length), _stream(stream, self.device)))
        self.n_tokens = int(queries.sum())
        return self

    def status(self) -> int:
        """Waits for the device; raises if a kernel of this batch gave up, or met a position outside the rotation's table."""
        v = _i64()
        _check(self._lib.httm_batch_status(self._handle(), ctypes.byref(v)))
        return int(v.value)


class KvCache:
    """Keys and values of one layer in pages: two tensors [pages][kv_heads][page_size][head_dim], bf16 or fp16, contiguous channels and any
    other strides ([pages][page_size][kv_heads][head_dim] as a permuted view, for instance)."""

    def __init__(self, k_pages: torch.Tensor, v_pages: torch.Tensor):
        self._lib = _library()
        for t, name in ((k_pages, "k_pages"), (v_pages, "v_pages")):
            if not t.is_cuda or t.dim() != 4 or t.stride(3) != 1 or t.dtype not in _DTYPES:
                _bad(f"{name}: expected a CUDA bfloat16 or float16 tensor [pages][kv_heads][page_size][head_dim] with contiguous channels")
        if k_pages.shape != v_pages.shape or k_pages.dtype != v_pages.dtype or k_pages.device != v_pages.device:
            _bad("k_pages and v_pages must have the same shape, type and device")
        self.k_pages, self.v_pages = k_pages, v_pages
        self.device = k_pages.get_device()
        self._dtype = k_pages.dtype
        self._in, self._in2, self._out = _Tensor(), _Tensor(), _Tensor()   # arguments of a call
        self._kind = _DTYPES[k_pages.dtype]
        self._pages = [_Pages(t.data_ptr(), t.stride(0), t.stride(1), t.stride(2)) for t in (k_pages, v_pages)]

        self._shape = tuple(k_pages.shape)

    def _check_batch(self, batch: CacheBatch):
        n, h, s, d = self._shape
        if h != batch.kv_heads or s != batch.page_size or d != batch.head_dim or n < batch.n_pages or batch.device != self.device:
            _bad("the batch is for caches of another shape or device")

    def append(self, batch: CacheBatch, k, v, rotary: Rotary = None, positions=None, k_weight=None, k_bias=None, stream=None):
        """The batch's tokens, k and v [kv_heads][tokens][head_dim], into their pages; with `rotary` keys are normed and rotated on the way,
        by `positions` or by the token's place behind the prefix."""
        self._check_batch(batch)
        shape = (batch.kv_heads, batch.n_tokens, batch.head_dim)
        tk, tv = self._in, self._in2
        tk.ptr, tk.stride_head, tk.stride_token = _rows(k, "k", shape, self._dtype, self.device)
        tv.ptr, tv.stride_head, tv.stride_token = _rows(v, "v", shape, self._dtype, self.device)
        pos = None
        if positions is not None:
            if rotary is None:
                _bad("positions without a rotary handle")
            pos = rotary._positions(positions, batch.n_tokens)
        _check(self._lib.httm_cache_append(batch._handle(), self._kind, self._pages[0], self._pages[1], tk, tv,
                                           None if rotary is None else rotary._handle(), pos, _vector(k_weight, "k_weight", batch.head_dim, self.device),
                                           _vector(k_bias, "k_bias", batch.head_dim, self.device), _stream(stream, self.device)))

    def attention(self, batch: CacheBatch, q, out=None, scale: float = None, stream=None) -> torch.Tensor:
        """q [heads][tokens][head_dim] against the prefix and each sequence's own keys; returns out [tokens][heads * head_dim]
        ([tokens][heads][head_dim] if `out` is given so).  scale: 1 / sqrt(head_dim) unless given."""
        self._check_batch(batch)
        H, N, D = batch.heads, batch.n_tokens, batch.head_dim
        tq, to = self._in, self._out
        tq.ptr, tq.stride_head, tq.stride_token = _rows(q, "q", (H, N, D), self._dtype, self.device)
        if out is None:
            out = torch.empty(N, H * D, dtype=self._dtype, device=q.device)
        if out.dtype is not self._dtype or out.get_device() != self.device:
            _bad("out: expected a CUDA tensor of q's type")
        strides = out.stride()
        if out.shape == (N, H * D) and strides[1] == 1:
            to.ptr, to.stride_head, to.stride_token = out.data_ptr(), D, strides[0]
        elif out.shape == (N, H, D) and strides[2] == 1:
            to.ptr, to.stride_head, to.stride_token = out.data_ptr(), strides[1], strides[0]
        else:
            _bad("out: expected [tokens][heads * head_dim] or [tokens][heads][head_dim] with contiguous channels")
        _check(self._lib.httm_cache_attention(batch._handle(), self._kind, self._pages[0], self._pages[1], tq, to,
                                              float(D ** -0.5 if scale is None else scale), _stream(stream, self.device)))
        return out
