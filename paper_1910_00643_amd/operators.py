"""Operators of a worker's local step for callers that keep their tensors in
PyTorch: a thin holder around include/slowmo_operators.h.  PyTorch supplies
device memory and the stream; all arithmetic on elements runs in libslowmo.so.

    Orthogonalizer   -- updates orthogonalised by Newton-Schulz products, alone or
                        behind the momentum of the SGD row of Table C.1
    HeadNormRotary   -- the norm of queries and keys for each head and the position
                        rotation, one pass, with its gradient
    rotary_table     -- the table of angles the rotation reads
"""
from __future__ import annotations

import ctypes as C
import struct
import threading
from typing import Optional, Sequence

import torch

from . import binding as B
from .optimizer import _DTYPE, _TORCH_GRAD, _raw_stream

SLOWMO_MAX_HEAD_DIM, SLOWMO_MAX_AXES, SLOWMO_MAX_ORTH_STEPS = 512, 4, 16
_SCALE = {"none": 0, "shape": 1, "rms": 2}

# every symbol include/slowmo_operators.h declares
EXPORTS = ["slowmo_head_norm_rotary", "slowmo_head_norm_rotary_backward", "slowmo_head_backward_bytes",
           "slowmo_orth_bytes", "slowmo_orth_create", "slowmo_orthogonalize",
           "slowmo_momentum_orthogonalize", "slowmo_orth_destroy"]


class slowmo_head_config(C.Structure):
    _fields_ = [("dtype", C.c_int32), ("head_dim", C.c_int32), ("rotary_dim", C.c_int32),
                ("interleaved", C.c_int32), ("norm", C.c_int32), ("eps", C.c_float),
                ("n_axes", C.c_int32), ("pair_axis", C.c_void_p), ("q_weight", C.c_void_p),
                ("k_weight", C.c_void_p), ("table", C.c_void_p), ("table_rows", C.c_int64),
                ("positions", C.c_void_p), ("position_stride", C.c_int64)]


class slowmo_heads(C.Structure):
    _fields_ = [("data", C.c_void_p), ("heads", C.c_int32), ("token_stride", C.c_int64),
                ("head_stride", C.c_int64)]


# the values of four and of six slowmo_heads side by side
_HEADS4, _HEADS6 = struct.Struct("@" + "Pi4xqq" * 4), struct.Struct("@" + "Pi4xqq" * 6)


class slowmo_orth_config(C.Structure):
    _fields_ = [("in_dtype", C.c_int32), ("out_dtype", C.c_int32), ("steps", C.c_int32),
                ("scale", C.c_int32), ("eps", C.c_float), ("coefficients", C.POINTER(C.c_float))]


_declared = None


def lib() -> C.CDLL:
    """The library with the operators' entry points declared."""
    global _declared
    if _declared is not None:
        return _declared
    L = B.lib()
    vp, i32, i64, size = C.c_void_p, C.c_int32, C.c_int64, C.c_size_t
    cfg, heads = C.POINTER(slowmo_head_config), C.POINTER(slowmo_heads)
    L.slowmo_head_norm_rotary.argtypes = [cfg, i64, heads, heads, heads, heads, vp, i64, vp]
    L.slowmo_head_norm_rotary_backward.argtypes = [cfg, i64, heads, heads, heads, heads, heads, heads,
                                                   vp, vp, vp, size, vp]
    L.slowmo_head_backward_bytes.argtypes = [cfg, i64, i32, i32]
    L.slowmo_head_backward_bytes.restype = size
    ocfg, list64, ptrs = C.POINTER(slowmo_orth_config), C.POINTER(i64), C.POINTER(vp)
    L.slowmo_orth_bytes.argtypes = [ocfg, i32, list64, list64, list64]
    L.slowmo_orth_bytes.restype = size
    L.slowmo_orth_create.argtypes = [C.POINTER(vp), ocfg, i32, list64, list64, list64, vp, size, vp]
    L.slowmo_orthogonalize.argtypes = [vp, ptrs, ptrs, vp]
    L.slowmo_momentum_orthogonalize.argtypes = [vp, ptrs, ptrs, ptrs, C.c_float, i32, vp]
    L.slowmo_orth_destroy.argtypes = [vp]
    _declared = L
    return L


def _check(status: int) -> None:
    if status != B.SLOWMO_OK:
        raise B.SlowMoError(status, B.slowmo_last_error(None))


# ---- norm of queries and keys with the position rotation ------------------------

def rotary_table(rows: int, pairs, base: float = 10000.0, device="cuda") -> torch.Tensor:
    """cos and sin of (position * base^(-i / n)) for positions 0..rows-1, as [rows, 2, pairs]
    fp32, computed in 64 bits.  `pairs`: the number of pairs, or, for several axes, how many
    each axis has: every axis then has frequencies of its own (i from 0 to n - 1)."""
    sections = [pairs] if isinstance(pairs, int) else list(pairs)
    freq = torch.cat([float(base) ** (-torch.arange(n, dtype=torch.float64) / n) for n in sections])
    angle = torch.arange(rows, dtype=torch.float64, device=device)[:, None] * freq.to(device)
    return torch.stack([angle.cos(), angle.sin()], 1).float().contiguous()


class _Arguments(threading.local):
    """The structures of a handle's calls, for each thread its own: ctypes lets go of the interpreter in a call."""

    def __init__(self, config):
        self.cfg = slowmo_head_config(**config)
        self.rows = (slowmo_heads * 6)()
        self.refs = [C.byref(r) for r in self.rows]


class HeadNormRotary:
    """The norm of queries and keys for each head and the position rotation.

    head_dim    -- elements of a head
    table       -- rotary_table(...), [rows, 2, pairs] fp32 on the GPU: the first 2 * pairs elements
                   of a head are turned; None: no rotation
    dtype       -- "bf16" or "f32": of queries, keys, results and their gradients
    norm, eps   -- whether to divide by sqrt(mean(x^2) + eps) and multiply by the weights (without it
                   a call has none)
    interleaved -- pair i is elements (2i, 2i + 1); else (i, i + pairs)
    pair_axis   -- the axis of positions that each pair belongs to; None: one axis

    Queries and keys are [tokens, heads, head_dim] (or with more leading dimensions that
    flatten without a copy), each head's elements contiguous, other strides free.
    `positions` is int64, [tokens] or [axes, tokens] (expanded, where all axes have the same): rows of the
    table, -1 for no turn.  A handle may serve several threads.  Calling it is an autograd function with a first
    derivative: no vmap, no forward mode, and torch.compile breaks its graph there."""

    def __init__(self, head_dim: int, table: Optional[torch.Tensor] = None, *, dtype: str = "bf16",
                 norm: bool = True, eps: float = 1e-6, interleaved: bool = False,
                 pair_axis: Optional[Sequence[int]] = None):
        pairs = 0
        if table is not None:
            assert table.dtype == torch.float32 and table.is_contiguous() and table.is_cuda
            assert table.dim() == 3 and table.shape[1] == 2
            pairs = table.shape[2]
        assert pair_axis is None or len(pair_axis) == pairs
        assert pair_axis is None or all(0 <= a < SLOWMO_MAX_AXES for a in pair_axis), "pair_axis: 0..3 for each pair"
        self.table, self.dtype, self.norm = table, _TORCH_GRAD[dtype], bool(norm)
        self.head_dim, self.pairs = int(head_dim), pairs
        self._axis = None if pair_axis is None else (C.c_uint8 * max(pairs, 1))(*pair_axis)
        self._args = _Arguments(dict(
            dtype=_DTYPE[dtype], head_dim=head_dim, rotary_dim=2 * pairs, interleaved=int(interleaved),
            norm=int(norm), eps=eps, n_axes=1,
            pair_axis=C.addressof(self._axis) if self._axis is not None else None,
            table=table.data_ptr() if table is not None else None,
            table_rows=table.shape[0] if table is not None else 0))

    # A call on few tokens ends before the next one is issued, so that the time between two launches is what
    # it takes: checks and addresses go straight into structures that the handle keeps, 10.8 -> 9.9 us a
    # call for 48 tokens.

    def _row(self, x: torch.Tensor, what: str):
        """The values of a slowmo_heads for [tokens, heads, head_dim]."""
        _, heads, dim = x.shape
        s0, s1, s2 = x.stride()
        assert x.dtype is self.dtype and x.is_cuda and dim == self.head_dim, what
        assert s2 == 1 or dim == 1 or x.numel() == 0, f"{what}: a head's elements must be contiguous"
        return x.data_ptr(), heads, s0, s1

    def _new(self, like: torch.Tensor):
        """A contiguous tensor for a result, and its slowmo_heads."""
        y = torch.empty_like(like, memory_format=torch.contiguous_format)
        heads, dim = like.shape[1], self.head_dim
        return y, (y.data_ptr(), heads, heads * dim, dim)

    def _weight(self, w):
        if w is None:
            return None
        assert w.dtype is torch.float32 and w.is_contiguous() and w.is_cuda and w.numel() == self.head_dim, \
            "weights: [head_dim] fp32"
        return w.data_ptr()

    def _config(self, positions, tokens, wq, wk) -> slowmo_head_config:
        cfg = self._args.cfg           # only what a call brings is written
        cfg.q_weight, cfg.k_weight = self._weight(wq), self._weight(wk)
        if self.pairs:
            shape, st = positions.shape, positions.stride()
            assert positions.dtype is torch.int64 and positions.is_cuda
            assert 0 < len(shape) < 3 and shape[-1] == tokens and (tokens < 2 or st[-1] == 1), \
                "positions: [tokens] or [axes, tokens], an axis's tokens contiguous"
            if len(shape) == 2 and shape[0] != 1:
                cfg.n_axes, cfg.position_stride = shape[0], st[0]
            else:
                cfg.n_axes, cfg.position_stride = 1, 0
            cfg.positions = positions.data_ptr()
        return cfg

    @staticmethod
    def _flat(x):
        return x if x.dim() == 3 else x.view(-1, x.shape[-2], x.shape[-1])

    def forward(self, q, k, positions=None, q_weight=None, k_weight=None, q_out=None, k_out=None,
                k_slots=None):
        """(turned queries, turned keys); written to q_out and k_out where given (they may be q
        and k).  With k_slots (int64, [tokens]), token t's keys go to row k_slots[t] of k_out,
        [rows, heads, head_dim], and to none where that lies outside it."""
        shapes = q.shape, k.shape
        q, k = self._flat(q), self._flat(k)
        tokens = rows = q.shape[0]
        assert k.shape[0] == tokens
        at_q, at_k = self._row(q, "q"), self._row(k, "k")
        if q_out is None:
            yq, at_yq = self._new(q)
        else:
            yq = self._flat(q_out)
            assert yq.shape == q.shape
            at_yq = self._row(yq, "q_out")
        slots = None
        if k_out is None:
            assert k_slots is None
            yk, at_yk = self._new(k)
        else:
            yk = self._flat(k_out)
            if k_slots is None:
                assert yk.shape == k.shape
            else:
                assert k_slots.dtype is torch.int64 and k_slots.is_contiguous()
                assert k_slots.is_cuda and k_slots.numel() == tokens
                slots, rows = k_slots.data_ptr() or None, yk.shape[0]
            at_yk = self._row(yk, "k_out")
        cfg = self._config(positions, tokens, q_weight, k_weight)
        _HEADS4.pack_into(self._args.rows, 0, *at_q, *at_k, *at_yq, *at_yk)
        r = self._args.refs
        status = lib().slowmo_head_norm_rotary(cfg, tokens, r[0], r[1], r[2], r[3], slots, rows,
                                               _raw_stream(q.device) or None)
        if status:
            _check(status)
        return ((yq if len(shapes[0]) == 3 else yq.view(shapes[0])) if q_out is None else q_out,
                (yk if len(shapes[1]) == 3 else yk.view(shapes[1])) if k_out is None else k_out)

    def backward(self, gq, gk, q, k, positions=None, q_weight=None, k_weight=None):
        """(dq, dk, dq_weight, dk_weight) from the gradients of forward's results and its inputs;
        the last two are None without the norm."""
        shapes = q.shape, k.shape
        gq, gk, q, k = self._flat(gq), self._flat(gk), self._flat(q), self._flat(k)
        tokens, dev = q.shape[0], q.device
        assert gq.shape == q.shape and gk.shape == k.shape and k.shape[0] == tokens
        at_q, at_k = self._row(q, "q"), self._row(k, "k")
        (dq, at_dq), (dk, at_dk) = self._new(q), self._new(k)
        cfg = self._config(positions, tokens, q_weight, k_weight)
        dwq = dwk = space = None
        nbytes = 0
        if self.norm:
            dwq = torch.empty(self.head_dim, dtype=torch.float32, device=dev)
            dwk = torch.empty_like(dwq)
            nbytes = lib().slowmo_head_backward_bytes(cfg, tokens, at_q[1], at_k[1])
            space = torch.empty(nbytes, dtype=torch.uint8, device=dev)
        _HEADS6.pack_into(self._args.rows, 0, *self._row(gq, "gq"), *self._row(gk, "gk"), *at_q, *at_k, *at_dq, *at_dk)
        r = self._args.refs
        status = lib().slowmo_head_norm_rotary_backward(
            cfg, tokens, r[0], r[1], r[2], r[3], r[4], r[5],
            dwq.data_ptr() if self.norm else None, dwk.data_ptr() if self.norm else None,
            space.data_ptr() if nbytes else None, nbytes, _raw_stream(dev) or None)
        if status:
            _check(status)
        return (dq if len(shapes[0]) == 3 else dq.view(shapes[0]),
                dk if len(shapes[1]) == 3 else dk.view(shapes[1]), dwq, dwk)

    def __call__(self, q, k, positions=None, q_weight=None, k_weight=None):
        """forward() that autograd differentiates, for q, k and the weights."""
        return _HeadNormRotary.apply(self, q, k, positions, q_weight, k_weight)


class _HeadNormRotary(torch.autograd.Function):
    @staticmethod
    def forward(ctx, op, q, k, positions, q_weight, k_weight):
        ctx.op = op
        ctx.save_for_backward(q, k, positions, q_weight, k_weight)
        return op.forward(q, k, positions, q_weight, k_weight)

    @staticmethod
    @torch.autograd.function.once_differentiable
    def backward(ctx, gq, gk):
        q, k, positions, wq, wk = ctx.saved_tensors
        dq, dk, dwq, dwk = ctx.op.backward(gq.contiguous(), gk.contiguous(), q, k, positions, wq, wk)
        return (None, dq, dk, None, dwq if wq is not None else None, dwk if wk is not None else None)


# ---- orthogonalised updates -------------------------------------------------------

class Orthogonalizer:
    """Orthogonalises a list of matrices by Newton-Schulz products.

    shapes       -- (rows, cols) of every tensor, or (count, rows, cols) for a stack of
                    matrices (the experts of a layer); convolutions as (outputs, inputs * window)
    dtype        -- "bf16" or "f32": of the tensors read
    out_dtype    -- of the results (default: dtype); "bf16": products of halves, "f32": of pairs of halves
    steps, eps, coefficients -- as in slowmo_orth_config; coefficients: (a, b, c) for all
                    steps or one such triple for each
    scale        -- "none", "shape" or "rms" (slowmo_orth_scale)
    ld           -- elements from one row to the next for each tensor (default: cols)

    Tensors are contiguous (or, with ld, have that row stride and, in a stack, any distance
    between matrices); the workspace is allocated once, here."""

    def __init__(self, shapes, *, dtype: str = "bf16", out_dtype: Optional[str] = None, steps: int = 5,
                 eps: float = 1e-7, coefficients=None, scale: str = "none", ld=None, device="cuda"):
        self.shapes = [tuple(int(v) for v in s) for s in shapes]
        assert all(len(s) in (2, 3) for s in self.shapes)
        out_dtype = dtype if out_dtype is None else out_dtype
        self.dtype, self.out_dtype = _TORCH_GRAD[dtype], _TORCH_GRAD[out_dtype]
        self.device = torch.device(device)
        rows, cols, lds = [], [], []
        for j, s in enumerate(self.shapes):
            count = s[0] if len(s) == 3 else 1
            rows += [s[-2]] * count
            cols += [s[-1]] * count
            lds += [s[-1] if ld is None or ld[j] is None else int(ld[j])] * count
        self.ld = [s[-1] if ld is None or ld[j] is None else int(ld[j]) for j, s in enumerate(self.shapes)]
        self.n_matrices = len(rows)
        coef = None
        if coefficients is not None:
            flat = list(coefficients)
            triples = [flat] * steps if not isinstance(flat[0], (list, tuple)) else flat
            assert len(triples) == steps and all(len(t) == 3 for t in triples)
            coef = (C.c_float * (3 * steps))(*[float(v) for t in triples for v in t])
        cfg = slowmo_orth_config(in_dtype=_DTYPE[dtype], out_dtype=_DTYPE[out_dtype], steps=steps,
                                 scale=_SCALE[scale], eps=eps, coefficients=coef)
        n = max(self.n_matrices, 1)
        arrays = [(C.c_int64 * n)(*v) for v in (rows, cols, lds)]
        nbytes = lib().slowmo_orth_bytes(cfg, self.n_matrices, *arrays)
        if nbytes == 0:
            raise B.SlowMoError(B.SLOWMO_ERR_ARG, B.slowmo_last_error(None))
        with torch.cuda.device(self.device):
            self.workspace = torch.empty(nbytes, dtype=torch.uint8, device=self.device)
            self.device = self.workspace.device       # with its number, whichever was the current one
            self.handle = C.c_void_p()
            _check(lib().slowmo_orth_create(C.byref(self.handle), cfg, self.n_matrices, *arrays,
                                            self.workspace.data_ptr(), nbytes,
                                            torch.cuda.current_stream(self.device).cuda_stream or None))

    def pointer_array(self, tensors, dtype: torch.dtype):
        """ctypes array of every matrix's address (reusable for the same tensors)."""
        if len(tensors) != len(self.shapes):
            raise ValueError(f"{len(self.shapes)} tensors wanted, {len(tensors)} given")
        flat = []
        for t, s, ld in zip(tensors, self.shapes, self.ld):
            if tuple(t.shape) != s or t.dtype != dtype or t.device != self.device:
                raise ValueError(f"a {dtype} tensor of shape {s} on {self.device} is wanted: got {tuple(t.shape)}, "
                                 f"{t.dtype}, {t.device}")
            st = t.stride()
            if t.numel() and (s[-1] > 1 and st[-1] != 1 or s[-2] > 1 and st[-2] != ld):
                raise ValueError(f"rows must be contiguous and {ld} elements apart: strides are {st}")
            at = t.data_ptr()
            if len(s) == 2:
                flat.append(at if t.numel() else 0)
            else:
                step = st[0] * t.element_size()
                flat += [at + i * step if t.numel() else 0 for i in range(s[0])]
        return (C.c_void_p * max(len(flat), 1))(*flat)

    def _array(self, tensors, dtype):
        if not isinstance(tensors, C.Array):
            return self.pointer_array(tensors, dtype)
        if len(tensors) < self.n_matrices:
            raise ValueError(f"{self.n_matrices} addresses wanted, {len(tensors)} given")
        return tensors

    def orthogonalize(self, inputs, out) -> None:
        """out[i] <- the orthogonalised inputs[i]: lists of tensors, or arrays from
        pointer_array().  out may be inputs where the types are the same."""
        _check(lib().slowmo_orthogonalize(self.handle, self._array(inputs, self.dtype),
                                          self._array(out, self.out_dtype), _raw_stream(self.device) or None))

    def momentum_orthogonalize(self, grads, momentum, out, mu: float, nesterov: bool = True) -> None:
        """momentum <- mu momentum + grads (fp32, in place); out <- the orthogonalised
        grads + mu momentum (nesterov) or momentum.  What `out` holds goes to SlowMo.local_step
        as the gradient, with momentum 0 there.  The momentum stays the caller's: SlowMo's buffer
        policies, averages and export_state() do not reach it (zero it after an outer step to reset it)."""
        _check(lib().slowmo_momentum_orthogonalize(
            self.handle, self._array(grads, self.dtype), self._array(momentum, torch.float32),
            self._array(out, self.out_dtype), mu, int(nesterov), _raw_stream(self.device) or None))

    def close(self) -> None:
        if getattr(self, "handle", None):
            torch.cuda.synchronize(self.device)
            lib().slowmo_orth_destroy(self.handle)
            self.handle = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass
