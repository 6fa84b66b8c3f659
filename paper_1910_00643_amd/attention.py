"""Attention for callers that keep their tensors in PyTorch: a thin holder around
include/slowmo_attention.h.  PyTorch supplies device memory and the stream; all
arithmetic on elements runs in libslowmo.so.

    Attention       -- over packed sequences, with a sliding window and first keys that
                       stay visible, forward and backward
    PagedAttention  -- new keys and values into a paged cache, turned by their positions,
                       and attention of the newest tokens over it
"""
from __future__ import annotations

import ctypes as C
from typing import Optional

import torch

from . import binding as B
from .operators import _check, slowmo_heads
from .optimizer import _DTYPE, _TORCH_GRAD, _raw_stream

SLOWMO_MAX_ATTENTION_DIM, SLOWMO_MAX_PAGE = 256, 65536

# every symbol include/slowmo_attention.h declares
EXPORTS = ["slowmo_attention", "slowmo_attention_backward", "slowmo_attention_backward_bytes", "slowmo_cache_append",
           "slowmo_paged_attention", "slowmo_paged_attention_bytes"]


class slowmo_attention_config(C.Structure):
    _fields_ = [("dtype", C.c_int32), ("head_dim", C.c_int32), ("causal", C.c_int32), ("clear_rest", C.c_int32),
                ("scale", C.c_float), ("window", C.c_int64), ("sinks", C.c_int64)]


class slowmo_cache(C.Structure):
    _fields_ = [("data", C.c_void_p), ("heads", C.c_int32), ("page", C.c_int32), ("pages", C.c_int64),
                ("page_stride", C.c_int64), ("token_stride", C.c_int64), ("head_stride", C.c_int64)]


class slowmo_pages(C.Structure):
    _fields_ = [("batch", C.c_int32), ("columns", C.c_int32), ("stride", C.c_int64), ("pages", C.c_void_p),
                ("lengths", C.c_void_p), ("offsets", C.c_void_p)]


class slowmo_append_config(C.Structure):
    _fields_ = [("dtype", C.c_int32), ("head_dim", C.c_int32), ("rotary_dim", C.c_int32), ("interleaved", C.c_int32),
                ("clear_rest", C.c_int32), ("table", C.c_void_p), ("table_rows", C.c_int64)]


_declared = None


def lib() -> C.CDLL:
    """The library with the attention's entry points declared."""
    global _declared
    if _declared is not None:
        return _declared
    L = B.lib()
    vp, i32, i64, size = C.c_void_p, C.c_int32, C.c_int64, C.c_size_t
    cfg, heads = C.POINTER(slowmo_attention_config), C.POINTER(slowmo_heads)
    pages, cache = C.POINTER(slowmo_pages), C.POINTER(slowmo_cache)
    L.slowmo_attention.argtypes = [cfg, i32, vp, vp, i64, i64, heads, heads, heads, heads, vp, vp]
    L.slowmo_attention_backward_bytes.argtypes = [cfg, i32, i64, i64, i32, i32]
    L.slowmo_attention_backward_bytes.restype = size
    L.slowmo_attention_backward.argtypes = [cfg, i32, vp, vp, i64, i64] + [heads] * 5 + [vp] + [heads] * 3 + [vp, size, vp]
    L.slowmo_cache_append.argtypes = [C.POINTER(slowmo_append_config), pages, i64, heads, heads, cache, cache, heads,
                                      heads, vp]
    L.slowmo_paged_attention_bytes.argtypes = [cfg, pages, i64, i32, cache]
    L.slowmo_paged_attention_bytes.restype = size
    L.slowmo_paged_attention.argtypes = [cfg, pages, i64, heads, cache, cache, heads, vp, vp, size, vp]
    _declared = L
    return L


class _Holder:
    """What both kinds of attention check of their tensors."""

    def __init__(self, head_dim: int, dtype: str):
        self.head_dim, self.dtype = int(head_dim), _TORCH_GRAD[dtype]

    def _rows(self, x: torch.Tensor, what: str, device: torch.device) -> slowmo_heads:
        """A slowmo_heads for [tokens, heads, head_dim]."""
        if x.dim() != 3 or x.shape[2] != self.head_dim or x.dtype is not self.dtype or x.device != device:
            raise ValueError(f"{what}: a {self.dtype} tensor [tokens, heads, {self.head_dim}] on {device} is wanted: got "
                             f"{tuple(x.shape)}, {x.dtype}, {x.device}")
        s0, s1, s2 = x.stride()
        if s2 != 1 and self.head_dim != 1 and x.numel():
            raise ValueError(f"{what}: a head's elements must be contiguous")
        return slowmo_heads(x.data_ptr(), x.shape[1], s0, s1)

    @staticmethod
    def _list(x: torch.Tensor, what: str, device: torch.device, length: Optional[int] = None) -> int:
        if x.dim() != 1 or x.dtype is not torch.int64 or not x.is_contiguous() or x.device != device or \
                x.shape[0] != (x.shape[0] if length is None else length):
            raise ValueError(f"{what}: a contiguous int64 tensor of {'[batch + 1]' if length is None else [length]} on {device} "
                             f"is wanted: got {tuple(x.shape)}, {x.dtype}, {x.device}")
        if not x.shape[0] and length is None:
            raise ValueError(f"{what}: batch + 1 entries are wanted")
        return x.data_ptr()

    @staticmethod
    def _device(x: torch.Tensor) -> torch.device:
        if not x.is_cuda:
            raise ValueError("tensors on a GPU are wanted")
        return x.device

    def _config(self, dtype, scale, causal, window, sinks) -> dict:
        window, sinks = int(window or 0), int(sinks)
        return dict(dtype=_DTYPE[dtype], head_dim=self.head_dim, causal=int(bool(causal)),
                    scale=float(self.head_dim) ** -0.5 if scale is None else scale, window=window, sinks=sinks)


class Attention(_Holder):
    """softmax(scale q k^T) v over packed sequences.

    head_dim    -- elements of a head, 1..256
    dtype       -- "bf16" or "f32": of queries, keys, values, results and gradients
    scale       -- of the products (default: head_dim ** -0.5)
    causal      -- a query sees the keys up to its own position only
    window      -- a query sees keys less than `window` positions away; None: any
    sinks       -- the first `sinks` keys of a sequence stay visible beside the window

    q is [tokens, heads, head_dim], k and v [keys, key heads, head_dim] (heads a multiple of key heads), a
    head's elements contiguous, other strides free.  `offsets`, int64 [batch + 1], ascending from 0, says where
    each sequence's rows begin; `k_offsets` the same for keys where they are other ones.  The last query of
    a sequence lies beside its last key.  Calling it is an autograd function with a first derivative: no vmap,
    no forward mode, and torch.compile breaks its graph there.  A handle may serve several threads."""

    def __init__(self, head_dim: int, *, dtype: str = "bf16", scale: Optional[float] = None, causal: bool = True,
                 window: Optional[int] = None, sinks: int = 0):
        super().__init__(head_dim, dtype)
        config = self._config(dtype, scale, causal, window, sinks)
        self._kept, self._cleared = (slowmo_attention_config(**config, clear_rest=c) for c in (0, 1))

    def _offsets(self, device, offsets, k_offsets):
        at = self._list(offsets, "offsets", device)
        batch = offsets.shape[0] - 1
        return batch, at, None if k_offsets is None else self._list(k_offsets, "k_offsets", device, batch + 1)

    def forward(self, q, k, v, offsets, k_offsets=None, out=None):
        """(out, lse): the result, written to `out` where given, and the logarithm of every query's sum of
        exponentials, fp32 [tokens, heads].  Rows behind the last sequence: of `out`, where given, left as they are;
        otherwise zeros.  lse there: -infinity."""
        device = self._device(q)
        rq, rk, rv = self._rows(q, "q", device), self._rows(k, "k", device), self._rows(v, "v", device)
        if v.shape[0] != k.shape[0]:
            raise ValueError("k and v must have the same number of rows")
        batch, at, k_at = self._offsets(device, offsets, k_offsets)
        fresh = out is None
        with torch.cuda.device(device):
            if fresh:
                out = torch.empty_like(q, memory_format=torch.contiguous_format)
            elif out.shape != q.shape:
                raise ValueError("out must have q's shape")
            lse = torch.empty(q.shape[:2], dtype=torch.float32, device=device)
            if not fresh:
                lse.fill_(float("-inf"))
            _check(lib().slowmo_attention(self._cleared if fresh else self._kept, batch, at, k_at, q.shape[0], k.shape[0], rq,
                                          rk, rv, self._rows(out, "out", device), lse.data_ptr() or None,
                                          _raw_stream(device) or None))
        return out, lse

    def backward(self, g, q, k, v, out, lse, offsets, k_offsets=None):
        """(dq, dk, dv) from the gradient of forward's result, its inputs and what it returned."""
        device = self._device(q)
        rows = [self._rows(x, n, device) for x, n in ((g, "g"), (q, "q"), (k, "k"), (v, "v"), (out, "out"))]
        if g.shape != q.shape or out.shape != q.shape or v.shape != k.shape:
            raise ValueError("g and out must have q's shape, v must have k's")
        if lse.shape != q.shape[:2] or lse.dtype is not torch.float32 or not lse.is_contiguous() or lse.device != device:
            raise ValueError("lse: what forward returned is wanted")
        batch, at, k_at = self._offsets(device, offsets, k_offsets)
        with torch.cuda.device(device):
            new = [torch.empty_like(x, memory_format=torch.contiguous_format) for x in (q, k, v)]
            nbytes = lib().slowmo_attention_backward_bytes(self._cleared, batch, q.shape[0], k.shape[0], q.shape[1], k.shape[1])
            space = torch.empty(nbytes, dtype=torch.uint8, device=device)
            _check(lib().slowmo_attention_backward(
                self._cleared, batch, at, k_at, q.shape[0], k.shape[0], *rows, lse.data_ptr() or None,
                *[self._rows(x, "a gradient", device) for x in new], space.data_ptr() if nbytes else None, nbytes,
                _raw_stream(device) or None))
        return tuple(new)

    def __call__(self, q, k, v, offsets, k_offsets=None):
        """forward()'s result, which autograd differentiates for q, k and v."""
        return _Attention.apply(self, q, k, v, offsets, k_offsets)


class _Attention(torch.autograd.Function):
    @staticmethod
    def forward(ctx, op, q, k, v, offsets, k_offsets):
        ctx.op = op
        out, lse = op.forward(q, k, v, offsets, k_offsets)
        ctx.save_for_backward(q, k, v, out, lse, offsets, k_offsets)
        return out

    @staticmethod
    @torch.autograd.function.once_differentiable
    def backward(ctx, g):
        q, k, v, out, lse, offsets, k_offsets = ctx.saved_tensors
        if g.stride(-1) != 1:
            g = g.contiguous()
        dq, dk, dv = ctx.op.backward(g, q, k, v, out, lse, offsets, k_offsets)
        return None, dq, dk, dv, None, None


class PagedAttention(_Holder):
    """New keys and values into a paged cache, and attention of each sequence's newest tokens over it.

    head_dim    -- elements of a head, 1..256
    table       -- rotary_table(...), [rows, 2, pairs] fp32 on the GPU: append turns the first 2 * pairs elements
                   of a key (and query) by the row of its position; None: it turns nothing
    interleaved -- pair i is elements (2i, 2i + 1); else (i, i + pairs)
    dtype, scale, window, sinks -- as Attention has them; a query sees no position after its own

    The caches are [pages, page, heads, head_dim], a head's elements contiguous, other strides free, `page` a power
    of two.  `pages`, int32 [batch, columns], a row's entries contiguous: the pages of each sequence in their order
    (entries that no position needs may hold anything); `lengths`, int64 [batch]: positions of each sequence, the
    new tokens, which are its last ones, included; `offsets`, int64 [batch + 1], ascending from 0: where each
    sequence's new tokens begin in q, k and v.  A handle may serve several threads."""

    def __init__(self, head_dim: int, table: Optional[torch.Tensor] = None, *, dtype: str = "bf16",
                 interleaved: bool = False, scale: Optional[float] = None, window: Optional[int] = None, sinks: int = 0):
        super().__init__(head_dim, dtype)
        pairs = 0
        if table is not None:
            if table.dtype is not torch.float32 or not table.is_contiguous() or not table.is_cuda or table.dim() != 3 or \
                    table.shape[1] != 2:
                raise ValueError("table: [rows, 2, pairs] fp32 on a GPU, contiguous, is wanted")
            pairs = table.shape[2]
        self.table = table
        self._cfg = slowmo_attention_config(**self._config(dtype, scale, True, window, sinks), clear_rest=0)
        self._cleared = slowmo_attention_config(**self._config(dtype, scale, True, window, sinks), clear_rest=1)
        self._append, self._append_cleared = (slowmo_append_config(
            dtype=_DTYPE[dtype], head_dim=self.head_dim, rotary_dim=2 * pairs, interleaved=int(bool(interleaved)), clear_rest=c,
            table=table.data_ptr() if pairs else None, table_rows=table.shape[0] if pairs else 0) for c in (0, 1))

    def _cache(self, x: torch.Tensor, what: str, device) -> slowmo_cache:
        if x.dim() != 4 or x.shape[3] != self.head_dim or x.dtype is not self.dtype or x.device != device:
            raise ValueError(f"{what}: a {self.dtype} tensor [pages, page, heads, {self.head_dim}] on {device} is wanted: got "
                             f"{tuple(x.shape)}, {x.dtype}, {x.device}")
        s = x.stride()
        if s[3] != 1 and self.head_dim != 1 and x.numel():
            raise ValueError(f"{what}: a head's elements must be contiguous")
        return slowmo_cache(x.data_ptr(), x.shape[2], x.shape[1], x.shape[0], s[0], s[1], s[2])

    def _pages(self, pages, lengths, offsets, device) -> slowmo_pages:
        if pages.dim() != 2 or pages.dtype is not torch.int32 or pages.device != device or \
                (pages.shape[1] > 1 and pages.stride(1) != 1):
            raise ValueError(f"pages: an int32 tensor [batch, columns] on {device}, a row's entries contiguous, is wanted: got "
                             f"{tuple(pages.shape)}, {pages.dtype}, {pages.device}")
        batch, columns = pages.shape
        return slowmo_pages(batch, columns, max(pages.stride(0), columns), pages.data_ptr() or None,
                            self._list(lengths, "lengths", device, batch) or None,
                            self._list(offsets, "offsets", device, batch + 1))

    def append(self, k, v, k_cache, v_cache, pages, lengths, offsets, q=None, q_out=None):
        """Writes the new keys, turned, and values to their places.  With q: returns the turned queries, written to
        q_out where given (it may be q).  Rows behind the last sequence: of q_out, where given, left as they are;
        otherwise zeros."""
        device = self._device(k)
        rk, rv = self._rows(k, "k", device), self._rows(v, "v", device)
        if v.shape[0] != k.shape[0] or (q is not None and q.shape[0] != k.shape[0]):
            raise ValueError("q, k and v must have the same number of rows")
        if q is None and q_out is not None:
            raise ValueError("q_out without q")
        if self.table is not None and self.table.device != device:
            raise ValueError(f"the table is on {self.table.device}, the tensors on {device}")
        with torch.cuda.device(device):
            rq, rqo, cfg = None, None, self._append
            if q is not None:
                rq = self._rows(q, "q", device)
                if q_out is None:
                    cfg = self._append_cleared
                    q_out = torch.empty_like(q, memory_format=torch.contiguous_format)
                elif q_out.shape != q.shape:
                    raise ValueError("q_out must have q's shape")
                rqo = self._rows(q_out, "q_out", device)
            _check(lib().slowmo_cache_append(cfg, self._pages(pages, lengths, offsets, device), k.shape[0], rk, rv,
                                             self._cache(k_cache, "k_cache", device), self._cache(v_cache, "v_cache", device),
                                             rq, rqo, _raw_stream(device) or None))
        return q_out

    def forward(self, q, k_cache, v_cache, pages, lengths, offsets, out=None, return_lse: bool = False):
        """Attention of the new tokens' queries (turned already) over the cached positions, those of the new
        tokens included: out, or (out, lse).  Rows behind the last sequence: of `out`, where given, left as they
        are; otherwise zeros."""
        device = self._device(q)
        rq = self._rows(q, "q", device)
        ck, cv = self._cache(k_cache, "k_cache", device), self._cache(v_cache, "v_cache", device)
        pg = self._pages(pages, lengths, offsets, device)
        cfg = self._cfg
        with torch.cuda.device(device):
            if out is None:
                cfg, out = self._cleared, torch.empty_like(q, memory_format=torch.contiguous_format)
            elif out.shape != q.shape:
                raise ValueError("out must have q's shape")
            lse = torch.full(q.shape[:2], float("-inf"), dtype=torch.float32, device=device) if return_lse else None
            nbytes = lib().slowmo_paged_attention_bytes(cfg, pg, q.shape[0], q.shape[1], ck)
            space = torch.empty(nbytes, dtype=torch.uint8, device=device) if nbytes else None
            _check(lib().slowmo_paged_attention(cfg, pg, q.shape[0], rq, ck, cv, self._rows(out, "out", device),
                                                lse.data_ptr() or None if return_lse else None,
                                                space.data_ptr() if nbytes else None, nbytes, _raw_stream(device) or None))
        return (out, lse) if return_lse else out

    __call__ = forward
