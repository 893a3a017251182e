"""Attention operators (C ABI in include/tcu_attn.h): the norm of each head of
queries and keys with the rotation by position, and attention over a sliding
window and a sequence's first tokens; over prompts, with their gradients, and
for one token.

Rows are torch tensors as the sequence operators take them (sequence.py), with
heads: dense -- (batch, length, heads, dim) -- or packed: (rows, heads, dim) with
``offsets``.  Any strides over batch and rows are taken as they are; a row's
values must be adjacent.  ``norm_rotate`` takes float32, bfloat16 and float16,
attention bfloat16 and float16, in rows that start at multiples of 16 bytes and
do not overlap.  Streams, ``out`` and autograd are as there: ``norm_rotate`` and
``window_attention`` record themselves where a gradient is asked of an argument;
the ``_grad`` calls are what that runs; the calls on caches have no gradient.
"""
from __future__ import annotations

import ctypes
import math
import struct
import threading
from collections import namedtuple

import torch
from torch.autograd import forward_ad as _forward

from . import OK, TcuDftError, lib
from .sequence import (_NO_ROWS, _TYPES, _apart, _flat, _grouped_rows, _i32, _i64, _no_grad,
                       _no_tangent, _On, _Rows, _tensor, _vp, _wants_grad, _written)

MAX_NORM_DIM = 256
MAX_DIM = 128

SYMBOLS = (
    "tcu_norm_rotate", "tcu_norm_rotate_grad", "tcu_norm_rotate_grad_workspace",
    "tcu_window_attention", "tcu_window_attention_grad", "tcu_window_attention_grad_workspace",
    "tcu_window_attention_step", "tcu_window_cache",
)

RotateGrads = namedtuple("RotateGrads", "q k q_weight k_weight")
AttentionGrads = namedtuple("AttentionGrads", "q k v")

_f32 = ctypes.c_float


class _RotateArgs(ctypes.Structure):
    _fields_ = [("type", _i32), ("sequences", _i32), ("heads", _i32), ("kv_heads", _i32),
                ("dim", _i32), ("turned", _i32), ("interleaved", _i32), ("eps", _f32),
                ("rows", _i64), ("offsets", _vp), ("positions", _vp),
                ("q", _Rows), ("k", _Rows), ("y_q", _Rows), ("y_k", _Rows),
                ("rates", _vp), ("q_weight", _vp), ("k_weight", _vp),
                ("dy_q", _Rows), ("dy_k", _Rows), ("dq", _Rows), ("dk", _Rows),
                ("dq_weight", _vp), ("dk_weight", _vp),
                ("workspace", _vp), ("workspace_bytes", _i64)]


class _AttentionArgs(ctypes.Structure):
    _fields_ = [("type", _i32), ("sequences", _i32), ("heads", _i32), ("kv_heads", _i32),
                ("dim", _i32), ("window", _i32), ("sinks", _i32), ("scale", _f32),
                ("rows", _i64), ("offsets", _vp),
                ("q", _Rows), ("k", _Rows), ("v", _Rows), ("y", _Rows), ("lse", _vp),
                ("dy", _Rows), ("dq", _Rows), ("dk", _Rows), ("dv", _Rows),
                ("workspace", _vp), ("workspace_bytes", _i64),
                ("cache_k", _vp), ("cache_v", _vp), ("slots", _vp), ("positions", _vp),
                ("num_slots", _i64)]


_ROTATE = struct.Struct("7ifq2P" + "P2q" * 4 + "3P" + "P2q" * 4 + "2P" + "Pq")
_ATTEND = struct.Struct("7ifqP" + "P2q" * 4 + "P" + "P2q" * 4 + "Pq" + "4P" + "q")
assert _ROTATE.size == ctypes.sizeof(_RotateArgs) and _ATTEND.size == ctypes.sizeof(_AttentionArgs)

_bound = None
_calls = {}
_binding = threading.Lock()


def _lib():
    global _bound, _calls
    if _bound is None:
        with _binding:
            if _bound is None:
                L, calls = lib(), {}
                for name in SYMBOLS:
                    f = getattr(L, name)
                    args = ctypes.POINTER(_RotateArgs if "rotate" in name else _AttentionArgs)
                    f.argtypes = [args] if name.endswith("workspace") else [args, _vp]
                    f.restype = _i64 if name.endswith("workspace") else ctypes.c_int
                    f = calls[name] = L[name]  # the same entry, for packed arguments
                    f.argtypes = ([ctypes.c_char_p] if name.endswith("workspace")
                                  else [ctypes.c_char_p, _vp])
                    f.restype = _i64 if name.endswith("workspace") else ctypes.c_int
                # published whole: other threads look entries up without the lock
                _calls = calls
                _bound = L
    return _bound


def _entry(name):
    f = _calls.get(name)
    if f is None:
        _lib()
        f = _calls[name]
    return f


def _call(name, packed, stream):
    rc = _entry(name)(packed, stream)
    if rc != OK:
        raise TcuDftError(rc, name)


def _workspace(name, packed, device):
    n = _entry(name)(packed)
    if n < 0:
        raise TcuDftError(2, name)
    return torch.empty(n, dtype=torch.uint8, device=device) if n else None, n


def _heads(q, k, offsets, types, what, loose=False, name="q"):
    """(sequences, rows, heads, key heads, dim, address of offsets, shapes of
    q and k); loose: three dimensions are rows even without offsets; name: q's."""
    _tensor(q, name)
    _tensor(k, "k")
    if q.dtype not in types:
        raise TypeError("%s must be %s" % (name, what))
    if not q.is_cuda:
        raise ValueError("%s must be a CUDA tensor" % name)
    shape = q.shape
    flat = offsets is not None or (loose and len(shape) == 3)
    if len(shape) != (3 if flat else 4):
        raise ValueError("%s must be (batch, length, heads, dim), or (rows, heads, dim) with "
                         "offsets" % name)
    heads, dim = shape[-2:]
    if k.dim() != len(shape):
        raise ValueError("k must have %d dimensions, as q" % len(shape))
    kv = k.shape[-2]
    if heads < 1 or kv < 1:
        raise ValueError("q and k must have one head at least")
    off = 0
    if offsets is not None:
        _tensor(offsets, "offsets")
        if (offsets.dtype != torch.int32 or offsets.device != q.device or offsets.dim() != 1
                or offsets.shape[0] < 1 or not offsets.is_contiguous()):
            raise ValueError("offsets must be a contiguous int32 tensor of sequences + 1 "
                             "values on %s" % q.device)
        off = offsets.data_ptr()
    seqs = offsets.shape[0] - 1 if offsets is not None else 1 if flat else shape[0]
    return seqs, shape[0] if flat else shape[1], heads, kv, dim, off, shape, shape[:-2] + (kv, dim)


def _beside(t):
    """t with the values of a row next to each other, as gradients come in."""
    st, sh = t.stride(), t.shape
    if (st[-1] == 1 or sh[-1] == 1) and (st[-2] == sh[-1] or sh[-2] == 1):
        return t
    return t.contiguous()


# ----------------------------------------------------------- norm and rotation
class _RotateCall:
    """The checked arguments that the operator and its gradient share."""

    def __init__(self, q, k, rates, q_weight, k_weight, positions, offsets, eps, interleaved):
        seqs, rows, heads, kv, dim, off, qs, ks = _heads(
            q, k, offsets, _TYPES, "float32, bfloat16 or float16", loose=True)
        if offsets is None and positions is None and q.dim() == 3:
            raise ValueError("rows without a batch need positions or offsets")
        dtype, index, f32 = q.dtype, q.get_device(), torch.float32
        if dim % 2 or not 2 <= dim <= MAX_NORM_DIM:
            raise ValueError("heads must have an even number of values up to %d" % MAX_NORM_DIM)
        _tensor(rates, "rates")
        if rates.dim() != 1 or not 1 <= rates.shape[0] <= dim // 2:
            raise ValueError("rates must be 1 to %d values" % (dim // 2))
        eps = float(eps)
        if not eps >= 0:
            raise ValueError("eps must not be negative")
        self.index, self.dtype, self.shapes, self.dim = index, dtype, (qs, ks), dim
        self.head = (_TYPES[dtype], seqs, heads, kv, dim, rates.shape[0], bool(interleaved), eps, rows,
                     off, _flat(positions, "positions", torch.int32, index, qs[:-2]),
                     *_grouped_rows(q, "q", dtype, index, qs), *_grouped_rows(k, "k", dtype, index, ks))
        self.params = (_flat(rates, "rates", f32, index, rates.shape),
                       _flat(q_weight, "q_weight", f32, index, (dim,)),
                       _flat(k_weight, "k_weight", f32, index, (dim,)))


def _rotate(q, k, rates, q_weight, k_weight, positions, offsets, eps, interleaved, out, stream):
    c = _RotateCall(q, k, rates, q_weight, k_weight, positions, offsets, eps, interleaved)
    with _On(c.index, stream) as st:
        qs, ks = c.shapes
        if out is None:
            yq = torch.empty(qs, dtype=c.dtype, device=q.device)
            yk = torch.empty(ks, dtype=c.dtype, device=q.device)
            ys = _fresh(yq, qs) + _fresh(yk, ks)
        else:
            yq, yk = out
            ys = (_grouped_rows(yq, "out", c.dtype, c.index, qs)
                  + _grouped_rows(yk, "out", c.dtype, c.index, ks))
            others = (rates, q_weight, k_weight, positions, offsets)
            _apart(yq, (k, *others), in_place=(q,))
            _apart(yk, (q, yq, *others), in_place=(k,))
        _call("tcu_norm_rotate", _ROTATE.pack(*c.head, *ys, *c.params, *_NO_ROWS * 4, 0, 0, 0, 0), st)
        if out is not None:
            _written(yq)
            _written(yk)
    return yq, yk


class _NormRotate(torch.autograd.Function):
    @staticmethod
    def forward(ctx, q, k, rates, q_weight, k_weight, positions, offsets, eps, interleaved):
        ctx.save_for_backward(q, k, rates, q_weight, k_weight, positions, offsets)
        ctx.eps, ctx.interleaved = eps, interleaved
        return _rotate(q, k, rates, q_weight, k_weight, positions, offsets, eps, interleaved, None,
                       None)

    @staticmethod
    @torch.autograd.function.once_differentiable
    def backward(ctx, dq, dk):
        q, k, rates, q_weight, k_weight, positions, offsets = ctx.saved_tensors
        g = norm_rotate_grad(_beside(dq), _beside(dk), q, k, rates, q_weight=q_weight,
                             k_weight=k_weight, positions=positions, offsets=offsets, eps=ctx.eps,
                             interleaved=ctx.interleaved)
        return g.q, g.k, None, g.q_weight, g.k_weight, None, None, None, None


def norm_rotate(q, k, rates, *, q_weight=None, k_weight=None, positions=None, offsets=None,
                eps=1e-6, interleaved=False, out=None, stream=None):
    """The norm of each head of queries and keys and their rotation by position:

        n = x / sqrt(mean(x^2) + eps) weight          (weights: (dim,), one if None)
        pairs (n[p], n[p + len(rates)]) turned by the angle position * rates[p]

    with ``interleaved`` the pairs (n[2p], n[2p + 1]); values from 2 len(rates)
    on are only normalised.  rates: float32, at most dim / 2; dim is even, at
    most 256.  positions: int32, one for each row; if None, the row's place in
    its sequence.  Rows (rows, heads, dim) go without offsets where positions
    are given: single tokens, for instance.

    Returns (q, k); ``out``, a pair, may be q and k themselves.  Angles are as
    exact at position 2^31 as at one, for rates up to 2^32.  Rows behind the last packed sequence are
    not written.
    """
    if _forward._current_level >= 0:
        _no_tangent(q, k, rates, q_weight, k_weight, *(out or ()))
    if _wants_grad(rates):
        raise ValueError("rates have no gradient")
    if _wants_grad(q, k, q_weight, k_weight):
        if out is not None or stream is not None:
            raise ValueError("out and stream cannot be given where a gradient is asked")
        return _NormRotate.apply(q, k, rates, q_weight, k_weight, positions, offsets, eps, interleaved)
    if out is not None:
        yq, yk = out
        if _wants_grad(yq, yk):
            raise ValueError("out must not record a gradient")
    return _rotate(q, k, rates, q_weight, k_weight, positions, offsets, eps, interleaved, out, stream)


def norm_rotate_grad(dq, dk, q, k, rates, *, q_weight=None, k_weight=None, positions=None,
                     offsets=None, eps=1e-6, interleaved=False, stream=None):
    """Gradients of norm_rotate's (q, k) under dq and dk: RotateGrads(q, k,
    q_weight, k_weight), None where the weight is.  Rows behind the last packed
    sequence get zeros."""
    if _forward._current_level >= 0:
        _no_tangent(dq, dk, q, k, rates, q_weight, k_weight)
    c = _RotateCall(q, k, rates, q_weight, k_weight, positions, offsets, eps, interleaved)
    dev, (qs, ks) = q.device, c.shapes
    pdy = (*_grouped_rows(dq, "dq", c.dtype, c.index, qs), *_grouped_rows(dk, "dk", c.dtype, c.index, ks))
    with _On(c.index, stream) as st:
        g = RotateGrads(*(torch.empty(s, dtype=c.dtype, device=dev) for s in c.shapes),
                        *(None if w is None else torch.empty(c.dim, dtype=torch.float32, device=dev)
                          for w in (q_weight, k_weight)))
        outs = (*_grouped_rows(g.q, "gradient", c.dtype, c.index, qs),
                *_grouped_rows(g.k, "gradient", c.dtype, c.index, ks),
                *(0 if w is None else w.data_ptr() for w in g[2:]))

        def packed(work, size):
            return _ROTATE.pack(*c.head, *_NO_ROWS * 2, *c.params, *pdy, *outs, work, size)

        work, n = _workspace("tcu_norm_rotate_grad_workspace", packed(0, 0), dev)
        _call("tcu_norm_rotate_grad", packed(work.data_ptr() if n else 0, n), st)
        del work
    return g


# ------------------------------------------------------------ window attention
_HALF = {torch.bfloat16: 1, torch.float16: 2}


def _rows16(t, name, dtype, index, shape):
    """_grouped_rows of rows that 16-byte accesses and tensor maps reach."""
    if not isinstance(t, torch.Tensor):
        _tensor(t, name)
    st, ptr = t.stride(), t.data_ptr()
    if len(st) == 4:
        batch, rows, heads, dim = shape
        b, r, h, d = st
    else:
        batch, (rows, heads, dim) = 1, shape
        b, (r, h, d) = 0, st if len(st) == 3 else (0, 0, 0)
    values = heads * dim
    if (t.dtype is dtype and t.shape == shape and t.get_device() == index and (h == dim or heads == 1)
            and d == 1 and ptr % 16 == 0 and (rows <= 1 or (r % 8 == 0 and r >= values))
            and (batch <= 1 or (b % 8 == 0 and b >= values))):
        return ptr, b, r
    r = _grouped_rows(t, name, dtype, index, shape)  # raises what is wrong
    if t.numel():
        raise ValueError("%s must hold its rows apart, each at a multiple of 16 bytes" % name)
    return r


def _fresh(t, shape):
    """A new tensor's rows."""
    row = shape[-1] * shape[-2]
    return (t.data_ptr(), shape[1] * row, row) if len(shape) == 4 else (t.data_ptr(), 0, row)


def _bounds(window, sinks, scale, dim):
    window, sinks = int(window), int(sinks)
    scale = dim ** -0.5 if scale is None else float(scale)
    if window < 1 or sinks < 0:
        raise ValueError("window must be 1 at least, and sinks not negative")
    if not (scale > 0 and math.isfinite(scale)):
        raise ValueError("scale must be positive")
    most = 2 ** 31 - 1  # beyond every row
    return min(window, most), min(sinks, most), scale


class _AttentionCall:
    """The checked arguments that the calls on rows share."""

    def __init__(self, q, k, v, window, sinks, scale, offsets, tokens=False, name="q"):
        seqs, rows, heads, kv, dim, off, qs, ks = _heads(q, k, offsets, _HALF, "bfloat16 or float16",
                                                         tokens, name)
        if heads % kv:
            raise ValueError("the %d heads of q must divide into the %d heads of k" % (heads, kv))
        if dim % 8 or not 8 <= dim <= MAX_DIM:
            raise ValueError("heads must have a multiple of 8 values up to %d" % MAX_DIM)
        dtype, index = q.dtype, q.get_device()
        window, sinks, scale = _bounds(window, sinks, scale, dim)
        self.index, self.dtype, self.shapes = index, dtype, (qs, ks)
        self.window, self.sinks, self.kv, self.dim = window, sinks, kv, dim
        self.sizes = (_HALF[dtype], seqs, heads, kv, dim, window, sinks, scale, rows, off)
        self.rows = (*_rows16(q, name, dtype, index, qs), *_rows16(k, "k", dtype, index, ks),
                     *_rows16(v, "v", dtype, index, ks))


_NO_GRAD_ROWS = _NO_ROWS * 4 + (0, 0)
_NO_CACHE = (0, 0, 0, 0, 0)


def _attend(q, k, v, window, sinks, scale, offsets, lse, out, stream):
    c = _AttentionCall(q, k, v, window, sinks, scale, offsets)
    with _On(c.index, stream) as st:
        if out is None:
            y = torch.empty(c.shapes[0], dtype=c.dtype, device=q.device)
            py = _fresh(y, c.shapes[0])
        else:
            y = out
            py = _rows16(y, "out", c.dtype, c.index, c.shapes[0])
            _apart(out, (q, k, v, offsets))
        sums = torch.empty(c.shapes[0][:-1], dtype=torch.float32, device=q.device) if lse else None
        _call("tcu_window_attention", _ATTEND.pack(*c.sizes, *c.rows, *py, sums.data_ptr() if lse else 0,
                                                   *_NO_GRAD_ROWS, *_NO_CACHE), st)
        if out is not None:
            _written(out)
    return y, sums


class _WindowAttention(torch.autograd.Function):
    @staticmethod
    def forward(ctx, q, k, v, window, sinks, scale, offsets):
        y, lse = _attend(q, k, v, window, sinks, scale, offsets, True, None, None)
        ctx.save_for_backward(q, k, v, y, lse, offsets)
        ctx.bounds = window, sinks, scale
        return y

    @staticmethod
    @torch.autograd.function.once_differentiable
    def backward(ctx, dy):
        q, k, v, y, lse, offsets = ctx.saved_tensors
        window, sinks, scale = ctx.bounds
        if dy.data_ptr() % 16 or any(s % 8 for n, s in zip(dy.shape[:-2], dy.stride()) if n > 1):
            dy = dy.clone(memory_format=torch.contiguous_format)
        elif any(s < dy.shape[-1] * dy.shape[-2] for n, s in zip(dy.shape[:-2], dy.stride()) if n > 1):
            dy = dy.contiguous()  # broadcast over rows
        g = window_attention_grad(_beside(dy), q, k, v, y, lse, window=window, sinks=sinks,
                                  scale=scale, offsets=offsets)
        return g.q, g.k, g.v, None, None, None, None


def window_attention(q, k, v, *, window, sinks=0, scale=None, offsets=None, lse=False, out=None,
                     stream=None):
    """Attention over a sliding window and a sequence's first tokens:

        y_i = sum_j p_ij v_j,  p_i = softmax of scale q_i.k_j over the visible j
        j visible to i: j <= i and (i - j < window or j < sinks)

    rows counted from their sequence's first.  q: (..., heads, dim); k, v: (...,
    key heads, dim), each serving heads / key heads adjacent heads of q; dim a
    multiple of 8 up to 128; scale: 1 / sqrt(dim) if None.  A window as long as
    the sequences is causal attention.

    Returns y, with ``lse`` also the log of each row's sum of exponentials
    (..., heads), which window_attention_grad takes.  Rows behind the last
    packed sequence are not written.  What is not finite reaches only the rows
    that see it; such a value of v may leave no number in all of their result.
    """
    if _forward._current_level >= 0:
        _no_tangent(q, k, v, out)
    if _wants_grad(q, k, v):
        if out is not None or lse or stream is not None:
            raise ValueError("out, lse and stream cannot be given where a gradient is asked")
        return _WindowAttention.apply(q, k, v, window, sinks, scale, offsets)
    if _wants_grad(out):
        raise ValueError("out must not record a gradient")
    y, sums = _attend(q, k, v, window, sinks, scale, offsets, lse, out, stream)
    return (y, sums) if lse else y


def window_attention_grad(dy, q, k, v, y, lse, *, window, sinks=0, scale=None, offsets=None,
                          stream=None):
    """Gradients of window_attention's y under dy, from y and the lse that it
    gave for the same arguments: AttentionGrads(q, k, v).  Rows behind the last
    packed sequence get zeros."""
    if _forward._current_level >= 0:
        _no_tangent(dy, q, k, v, y, lse)
    c = _AttentionCall(q, k, v, window, sinks, scale, offsets)
    dev, dtype, index, (qs, ks) = q.device, c.dtype, c.index, c.shapes
    py, pdy = _rows16(y, "y", dtype, index, qs), _rows16(dy, "dy", dtype, index, qs)
    pl = _flat(lse, "lse", torch.float32, index, qs[:-1])
    with _On(index, stream) as st:
        g = AttentionGrads(*(torch.empty(s, dtype=dtype, device=dev) for s in (qs, ks, ks)))
        outs = [x for t, s in zip(g, (qs, ks, ks)) for x in _rows16(t, "gradient", dtype, index, s)]

        def packed(work, size):
            return _ATTEND.pack(*c.sizes, *c.rows, *py, pl, *pdy, *outs, work, size, *_NO_CACHE)

        work, n = _workspace("tcu_window_attention_grad_workspace", packed(0, 0), dev)
        _call("tcu_window_attention_grad", packed(work.data_ptr() if n else 0, n), st)
        del work
    return g


def _caches(c, cache_k, cache_v, slots, batch):
    """(addresses of both caches, of slots, entries)."""
    _tensor(cache_k, "cache_k")
    if cache_k.dim() != 4:
        raise ValueError("cache_k must be (entries, sinks + window, key heads, dim)")
    n = cache_k.shape[0]
    shape = (n, c.window + c.sinks, c.kv, c.dim)
    pk = _flat(cache_k, "cache_k", c.dtype, c.index, shape)
    _tensor(cache_v, "cache_v")
    pv = _flat(cache_v, "cache_v", c.dtype, c.index, shape)
    if n and (pk % 16 or pv % 16):
        raise ValueError("caches must start at multiples of 16 bytes")
    if slots is None and n < batch:
        raise ValueError("the caches have %d entries for %d sequences" % (n, batch))
    return pk, pv, _flat(slots, "slots", torch.int32, c.index, (batch,)), n


def window_attention_step(q, k, v, cache_k, cache_v, positions, *, window, sinks=0, scale=None,
                          slots=None, out=None, stream=None):
    """window_attention for one more row of every sequence: q (batch, heads,
    dim), k, v (batch, key heads, dim), at positions (batch,), int32, to y.

    The caches (entries, sinks + window, key heads, dim) take k and v in place,
    at entry slots[b] (int32) for row b, or entry b: position p is row p of its
    entry if p < sinks, else row sinks + (p - sinks) % window.  A slot outside
    the caches or a position below zero gives a row of zeros; no two rows may
    name the same slot."""
    if _forward._current_level >= 0:
        _no_tangent(q, k, v, cache_k, cache_v, out)
    _no_grad(q, k, v, cache_k, cache_v, out)
    _tensor(q, "q")
    if q.dim() != 3:
        raise ValueError("q must be (batch, heads, dim)")
    c = _AttentionCall(q, k, v, window, sinks, scale, None, tokens=True)
    batch = q.shape[0]
    pk, pv, ps, n = _caches(c, cache_k, cache_v, slots, batch)
    if positions is None:
        _tensor(positions, "positions")
    pp = _flat(positions, "positions", torch.int32, c.index, (batch,))
    with _On(c.index, stream) as st:
        if out is None:
            y = torch.empty(c.shapes[0], dtype=c.dtype, device=q.device)
            py = _fresh(y, c.shapes[0])
        else:
            y = out
            py = _rows16(y, "out", c.dtype, c.index, c.shapes[0])
            _apart(out, (q, k, v, cache_k, cache_v, positions, slots))
        t, _, heads, kv, dim, w, s, scale = c.sizes[:8]
        r = c.rows
        _call("tcu_window_attention_step", _ATTEND.pack(
            t, batch, heads, kv, dim, w, s, scale, 1, 0, r[0], r[2], 0, r[3], r[5], 0, r[6], r[8], 0,
            py[0], py[2], 0, 0, *_NO_GRAD_ROWS, pk, pv, ps, pp, n), st)
        _written(cache_k)
        _written(cache_v)
        if out is not None:
            _written(out)
    return y


def window_cache(k, v, cache_k, cache_v, *, window, sinks=0, offsets=None, slots=None, stream=None):
    """Fills entries of the caches that window_attention_step takes from whole
    prompts k and v: of each sequence the rows that its next token sees, at
    entry slots[s] (int32) for sequence s, or entry s.  Other rows of the
    caches stay; slots outside them are passed over; no two sequences may name
    the same one."""
    if _forward._current_level >= 0:
        _no_tangent(k, v, cache_k, cache_v)
    _no_grad(k, v, cache_k, cache_v)
    c = _AttentionCall(k, k, v, window, sinks, 1.0, offsets, name="k")
    pk, pv, ps, n = _caches(c, cache_k, cache_v, slots, c.sizes[1])
    with _On(c.index, stream) as st:
        _call("tcu_window_cache", _ATTEND.pack(*c.sizes, *c.rows, *_NO_ROWS, 0, *_NO_GRAD_ROWS,
                                               pk, pv, ps, 0, n), st)
        _written(cache_k)
        _written(cache_v)
