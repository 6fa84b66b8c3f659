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
import struct
import threading
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


# the values of eight slowmo_heads side by side, of two slowmo_cache and of a slowmo_pages
_HEADS = [struct.Struct("@" + "Pi4xqq" * n) for n in range(9)]
_CACHES, _PAGES = struct.Struct("@" + "Piiqqqq" * 2), struct.Struct("@iiqPPP")


class _Arguments(threading.local):
    """The structures of a handle's calls, for each thread its own: ctypes lets go of the interpreter in a call."""

    def __init__(self):
        self.rows, self.caches, self.pages = (slowmo_heads * 8)(), (slowmo_cache * 2)(), slowmo_pages()
        self.row = [C.byref(r) for r in self.rows]
        self.k_cache, self.v_cache, self.table = C.byref(self.caches[0]), C.byref(self.caches[1]), C.byref(self.pages)


def _on(device: torch.device, call, *args):
    """The call with its tensors' GPU as the current one."""
    if torch.cuda.current_device() == device.index:
        status = call(*args)
    else:
        with torch.cuda.device(device):
            status = call(*args)
    if status:
        _check(status)


class _Holder:
    """What both kinds of attention check of their tensors.  A call on few tokens ends before the next one is issued,
    so that the time between two is what these checks take: addresses go straight into structures that the handle keeps."""

    def __init__(self, head_dim: int, dtype: str):
        self.head_dim, self.dtype = int(head_dim), _TORCH_GRAD[dtype]
        self._args = _Arguments()

    def _row(self, x: torch.Tensor, what: str, device: torch.device):
        """The values of a slowmo_heads for [tokens, heads, head_dim]."""
        shape = x.shape
        if len(shape) != 3 or shape[2] != self.head_dim or x.dtype is not self.dtype or x.device != device:
            raise ValueError(f"{what}: a {self.dtype} tensor [tokens, heads, {self.head_dim}] on {device} is wanted: got "
                             f"{tuple(shape)}, {x.dtype}, {x.device}")
        s0, s1, s2 = x.stride()
        if s2 != 1 and self.head_dim != 1 and x.numel():
            raise ValueError(f"{what}: a head's elements must be contiguous")
        return x.data_ptr(), shape[1], s0, s1

    def _rows(self, device, **tensors):
        """Fills the kept structures, one for each tensor in order."""
        values = []
        for what, x in tensors.items():
            values += self._row(x, what, device)
        _HEADS[len(tensors)].pack_into(self._args.rows, 0, *values)

    @staticmethod
    def _list(x: torch.Tensor, what: str, device: torch.device, length: Optional[int] = None) -> int:
        shape = x.shape
        if len(shape) != 1 or x.dtype is not torch.int64 or not x.is_contiguous() or x.device != device or \
                (length is not None and shape[0] != length) or (length is None and not shape[0]):
            raise ValueError(f"{what}: a contiguous int64 tensor of {'[batch + 1]' if length is None else [length]} on {device} "
                             f"is wanted: got {tuple(shape)}, {x.dtype}, {x.device}")
        return x.data_ptr()

    @staticmethod
    def _device(x: torch.Tensor) -> torch.device:
        if not x.is_cuda:
            raise ValueError("tensors on a GPU are wanted")
        return x.device

    def _config(self, dtype, scale, causal, window, sinks) -> dict:
        if window is not None and window < 1 or sinks < 0:
            raise ValueError("window must be at least 1, or None for any distance, and sinks at least 0")
        return dict(dtype=_DTYPE[dtype], head_dim=self.head_dim, causal=int(bool(causal)),
                    scale=float(self.head_dim) ** -0.5 if scale is None else scale,
                    # past every length; ctypes would keep the last 64 bits alone
                    window=min(int(window or 0), 1 << 62), sinks=min(int(sinks), 1 << 62))


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
        batch, at, k_at = self._offsets(device, offsets, k_offsets)
        cfg = self._kept
        if out is None:
            cfg, out = self._cleared, torch.empty_like(q, memory_format=torch.contiguous_format)
        if v.shape[0] != k.shape[0] or out.shape != q.shape:
            raise ValueError("k and v must have the same number of rows, out must have q's shape")
        self._rows(device, q=q, k=k, v=v, out=out)
        lse = torch.empty(q.shape[:2], dtype=torch.float32, device=device)
        if cfg is self._kept:
            lse.fill_(float("-inf"))
        r = self._args.row
        _on(device, lib().slowmo_attention, cfg, batch, at, k_at, q.shape[0], k.shape[0], r[0], r[1], r[2], r[3],
            lse.data_ptr() or None, _raw_stream(device) or None)
        return out, lse

    def backward(self, g, q, k, v, out, lse, offsets, k_offsets=None):
        """(dq, dk, dv) from the gradient of forward's result, its inputs and what it returned for them: `out` and `lse` of more
        keys than these, joined from several calls, are not meant, since dS of a row is taken to sum to 0."""
        device = self._device(q)
        if g.shape != q.shape or out.shape != q.shape or v.shape != k.shape:
            raise ValueError("g and out must have q's shape, v must have k's")
        if lse.shape != q.shape[:2] or lse.dtype is not torch.float32 or not lse.is_contiguous() or lse.device != device:
            raise ValueError("lse: what forward returned is wanted")
        batch, at, k_at = self._offsets(device, offsets, k_offsets)
        dq, dk, dv = (torch.empty_like(x, memory_format=torch.contiguous_format) for x in (q, k, v))
        self._rows(device, g=g, q=q, k=k, v=v, out=out, dq=dq, dk=dk, dv=dv)
        tokens, keys = q.shape[0], k.shape[0]
        nbytes = lib().slowmo_attention_backward_bytes(self._cleared, batch, tokens, keys, q.shape[1], k.shape[1])
        space = torch.empty(nbytes, dtype=torch.uint8, device=device)
        r = self._args.row
        _on(device, lib().slowmo_attention_backward, self._cleared, batch, at, k_at, tokens, keys, r[0], r[1], r[2], r[3], r[4],
            lse.data_ptr() or None, r[5], r[6], r[7], space.data_ptr() if nbytes else None, nbytes, _raw_stream(device) or None)
        return dq, dk, dv

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

    def _cache(self, x: torch.Tensor, what: str, device):
        shape = x.shape
        if len(shape) != 4 or shape[3] != self.head_dim or x.dtype is not self.dtype or x.device != device:
            raise ValueError(f"{what}: a {self.dtype} tensor [pages, page, heads, {self.head_dim}] on {device} is wanted: got "
                             f"{tuple(shape)}, {x.dtype}, {x.device}")
        s0, s1, s2, s3 = x.stride()
        if s3 != 1 and self.head_dim != 1 and x.numel():
            raise ValueError(f"{what}: a head's elements must be contiguous")
        return x.data_ptr(), shape[2], shape[1], shape[0], s0, s1, s2

    def _places(self, k_cache, v_cache, pages, lengths, offsets, device):
        """Fills the kept structures of the caches and of the table."""
        _CACHES.pack_into(self._args.caches, 0, *self._cache(k_cache, "k_cache", device),
                          *self._cache(v_cache, "v_cache", device))
        if pages.dim() != 2 or pages.dtype is not torch.int32 or pages.device != device or \
                (pages.shape[1] > 1 and pages.stride(1) != 1):
            raise ValueError(f"pages: an int32 tensor [batch, columns] on {device}, a row's entries contiguous, is wanted: got "
                             f"{tuple(pages.shape)}, {pages.dtype}, {pages.device}")
        batch, columns = pages.shape
        _PAGES.pack_into(self._args.pages, 0, batch, columns, pages.stride(0) if batch > 1 else columns, pages.data_ptr(),
                         self._list(lengths, "lengths", device, batch), self._list(offsets, "offsets", device, batch + 1))

    def append(self, k, v, k_cache, v_cache, pages, lengths, offsets, q=None, q_out=None):
        """Writes the new keys, turned, and values to their places.  With q: returns the turned queries, written to
        q_out where given (it may be q).  Rows behind the last sequence: of q_out, where given, left as they are;
        otherwise zeros."""
        device = self._device(k)
        if self.table is not None and self.table.device != device:
            raise ValueError(f"the table is on {self.table.device}, the tensors on {device}")
        cfg, r = self._append, self._args.row
        if q is None:
            if q_out is not None:
                raise ValueError("q_out without q")
            self._rows(device, k=k, v=v)
            tokens, rq, rqo = k.shape[0], None, None
        else:
            if q_out is None:
                cfg, q_out = self._append_cleared, torch.empty_like(q, memory_format=torch.contiguous_format)
            self._rows(device, k=k, v=v, q=q, q_out=q_out)
            tokens, rq, rqo = q.shape[0], r[2], r[3]
            if q_out.shape != q.shape:
                raise ValueError("q_out must have q's shape")
        if k.shape[0] != tokens or v.shape[0] != tokens:
            raise ValueError("q, k and v must have the same number of rows")
        self._places(k_cache, v_cache, pages, lengths, offsets, device)
        a = self._args
        _on(device, lib().slowmo_cache_append, cfg, a.table, tokens, r[0], r[1], a.k_cache, a.v_cache, rq, rqo,
            _raw_stream(device) or None)
        return q_out

    def forward(self, q, k_cache, v_cache, pages, lengths, offsets, out=None, return_lse: bool = False):
        """Attention of the new tokens' queries (turned already) over the cached positions, those of the new
        tokens included: out, or (out, lse).  Rows behind the last sequence: of `out`, where given, left as they
        are; otherwise zeros."""
        device = self._device(q)
        cfg = self._cfg
        if out is None:
            cfg, out = self._cleared, torch.empty_like(q, memory_format=torch.contiguous_format)
        self._rows(device, q=q, out=out)
        if out.shape != q.shape:
            raise ValueError("out must have q's shape")
        self._places(k_cache, v_cache, pages, lengths, offsets, device)
        lse = torch.full(q.shape[:2], float("-inf"), dtype=torch.float32, device=device) if return_lse else None
        a, tokens = self._args, q.shape[0]
        nbytes = lib().slowmo_paged_attention_bytes(cfg, a.table, tokens, q.shape[1], a.k_cache)
        space = torch.empty(nbytes, dtype=torch.uint8, device=device) if nbytes else None
        _on(device, lib().slowmo_paged_attention, cfg, a.table, tokens, a.row[0], a.k_cache, a.v_cache, a.row[1],
            lse.data_ptr() or None if return_lse else None, space.data_ptr() if nbytes else None, nbytes,
            _raw_stream(device) or None)
        return (out, lse) if return_lse else out

    __call__ = forward
