"""Sequence operators (C ABI in include/tcu_seq.h): the short causal
convolution, the selective state-space scan and the gated linear recurrence,
over prompts, with their gradients, and for one token.

Rows are torch tensors of float32, bfloat16 or float16, dense -- (batch,
length, channels) -- or packed: (rows, channels) with ``offsets``, an int32
CUDA tensor of sequences + 1 row numbers from 0 to rows.  Any strides over
batch and rows are taken as they are (a slice of a wider projection needs no
copy); channels must be adjacent.  Parameters and the states of scan and
recurrence are float32.  Everything runs on torch's current stream, or on ``stream``; ordering
that against other streams that use the tensors (wait_stream, record_stream) is
the caller's, as for any torch operation.  ``out``
shares memory neither with an input nor with itself; only a single-token call
may write over a row that it reads (x; u, dt or gate; forget or admit), all
of it.

``short_conv``, ``state_scan`` and ``gated_scan`` are differentiable: where a
gradient is asked of an argument they record themselves with autograd.  The ``_grad``
calls are what that runs; the ``_step`` calls have no gradient.
"""
from __future__ import annotations

import ctypes
import struct
import threading
from collections import namedtuple

import torch

from torch.autograd import forward_ad as _forward

from . import OK, TcuDftError, lib

MAX_WIDTH = 8
MAX_STATES = 128
MARK = 16  # rows from one state that the gradient resumes from to the next
GATED_MARK = 8  # the same for the gated recurrence

SYMBOLS = (
    "tcu_short_conv", "tcu_short_conv_grad", "tcu_short_conv_grad_workspace",
    "tcu_short_conv_step", "tcu_state_scan", "tcu_state_scan_workspace",
    "tcu_state_scan_grad", "tcu_state_scan_grad_workspace",
    "tcu_state_scan_step", "tcu_gated_scan", "tcu_gated_scan_workspace",
    "tcu_gated_scan_grad", "tcu_gated_scan_grad_workspace", "tcu_gated_scan_step",
)

_TYPES = {torch.float32: 0, torch.bfloat16: 1, torch.float16: 2}

ConvGrads = namedtuple("ConvGrads", "x weight bias state")
ScanGrads = namedtuple("ScanGrads", "u dt A B C skip gate dt_bias state")
GatedGrads = namedtuple("GatedGrads", "x forget admit rate state")

_vp, _i64, _i32 = ctypes.c_void_p, ctypes.c_int64, ctypes.c_int32


class _Rows(ctypes.Structure):
    _fields_ = [("ptr", _vp), ("batch_stride", _i64), ("row_stride", _i64)]


class _ConvArgs(ctypes.Structure):
    _fields_ = [("type", _i32), ("width", _i32), ("silu", _i32), ("sequences", _i32),
                ("rows", _i64), ("channels", _i64), ("offsets", _vp),
                ("x", _Rows), ("y", _Rows), ("dy", _Rows), ("dx", _Rows),
                ("weight", _vp), ("bias", _vp), ("state", _vp), ("dlast", _vp),
                ("last", _vp), ("dstate", _vp), ("dweight", _vp), ("dbias", _vp),
                ("workspace", _vp), ("workspace_bytes", _i64),
                ("slots", _vp), ("num_slots", _i64)]


class _ScanArgs(ctypes.Structure):
    _fields_ = [("type", _i32), ("softplus", _i32), ("sequences", _i32), ("groups", _i32),
                ("rows", _i64), ("channels", _i64), ("states", _i64), ("offsets", _vp),
                ("u", _Rows), ("dt", _Rows), ("gate", _Rows), ("y", _Rows), ("B", _Rows),
                ("C", _Rows),
                ("A", _vp), ("skip", _vp), ("dt_bias", _vp), ("state", _vp), ("dlast", _vp),
                ("last", _vp), ("dstate", _vp), ("marks", _vp),
                ("dy", _Rows), ("du", _Rows), ("ddt", _Rows), ("dgate", _Rows),
                ("dB", _Rows), ("dC", _Rows),
                ("dA", _vp), ("dskip", _vp), ("ddt_bias", _vp),
                ("workspace", _vp), ("workspace_bytes", _i64),
                ("slots", _vp), ("num_slots", _i64)]


class _GatedArgs(ctypes.Structure):
    _fields_ = [("type", _i32), ("sequences", _i32), ("rows", _i64), ("channels", _i64),
                ("offsets", _vp), ("x", _Rows), ("forget", _Rows), ("admit", _Rows), ("y", _Rows),
                ("rate", _vp), ("state", _vp), ("dlast", _vp),
                ("last", _vp), ("dstate", _vp), ("marks", _vp),
                ("dy", _Rows), ("dx", _Rows), ("dforget", _Rows), ("dadmit", _Rows),
                ("drate", _vp),
                ("workspace", _vp), ("workspace_bytes", _i64),
                ("slots", _vp), ("num_slots", _i64)]


# The same structures for struct.pack: what a call costs on the host counts
# where a token's kernel takes a few microseconds.
_CONV = struct.Struct("4i2qP" + "P2q" * 4 + "P" * 8 + "Pq" * 2)
_SCAN = struct.Struct("4i3qP" + "P2q" * 6 + "P" * 8 + "P2q" * 6 + "P" * 3 + "Pq" * 2)
_GATED = struct.Struct("2i2qP" + "P2q" * 4 + "P" * 6 + "P2q" * 4 + "P" + "Pq" * 2)
assert _CONV.size == ctypes.sizeof(_ConvArgs) and _SCAN.size == ctypes.sizeof(_ScanArgs)
assert _GATED.size == ctypes.sizeof(_GatedArgs)
_NO_ROWS = (0, 0, 0)

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
                    args = ctypes.POINTER(_ConvArgs if "conv" in name else
                                          _GatedArgs if "gated" in name else _ScanArgs)
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


def _call(name, packed, stream):
    f = _calls.get(name)
    if f is None:
        _lib()
        f = _calls[name]
    rc = f(packed, stream)
    if rc != OK:
        raise TcuDftError(rc, name)


_current_device = torch.cuda.current_device
_raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None) or (
    lambda index: torch.cuda.current_stream(index).cuda_stream)


class _On:
    """The device and stream of a call, current while it allocates and
    launches: memory that a call takes for itself belongs to its stream."""

    def __init__(self, index, stream):
        self.stream = stream
        self.index = index
        self.guards = ()
        if stream is not None and stream.device.index != index:
            raise ValueError("stream is of %s, the tensors are on cuda:%d" % (stream.device, index))
        if stream is not None or index != _current_device():
            self.guards = [torch.cuda.device(index)]
            if stream is not None:
                self.guards.append(torch.cuda.stream(stream))

    def __enter__(self):
        for g in self.guards:
            g.__enter__()
        return _raw_stream(self.index) if self.stream is None else self.stream.cuda_stream

    def __exit__(self, *exc):
        for g in reversed(self.guards):
            g.__exit__(*exc)


def _tensor(t, name):
    if not isinstance(t, torch.Tensor):
        raise TypeError("%s must be a torch tensor" % name)


def _wrong(t, name, dtype, index, shape, why):
    """Raises what is wrong with t."""
    _tensor(t, name)
    if t.dtype != dtype:
        raise TypeError("%s must be %s, not %s" % (name, dtype, t.dtype))
    if t.get_device() != index:
        raise ValueError("%s must be on cuda:%d, not %s" % (name, index, t.device))
    if t.shape != shape:
        raise ValueError("%s must have shape %s, not %s" % (name, tuple(shape), tuple(t.shape)))
    raise ValueError("%s must %s" % (name, why))


_ADJACENT = "hold the values of a row next to each other"


def _rows(t, name, dtype, index, shape):
    """t, (batch, rows, values) or (rows, values), as a row tensor: (pointer,
    batch stride, row stride)."""
    if not isinstance(t, torch.Tensor):
        _tensor(t, name)
    st = t.stride()
    if (t.dtype is not dtype or t.shape != shape or t.get_device() != index
            or (st[-1] != 1 and shape[-1] > 1)):
        _wrong(t, name, dtype, index, shape, _ADJACENT)
    return (t.data_ptr(), st[0], st[1]) if len(st) == 3 else (t.data_ptr(), 0, st[0])


def _grouped_rows(t, name, dtype, index, shape):
    """The same for (..., groups, states)."""
    if not isinstance(t, torch.Tensor):
        _tensor(t, name)
    st = t.stride()
    if (t.dtype is not dtype or t.shape != shape or t.get_device() != index
            or (st[-1] != 1 and shape[-1] > 1) or (st[-2] != shape[-1] and shape[-2] > 1)):
        _wrong(t, name, dtype, index, shape, _ADJACENT)
    return (t.data_ptr(), st[0], st[1]) if len(st) == 4 else (t.data_ptr(), 0, st[0])


def _flat(t, name, dtype, index, shape):
    """t as a contiguous array: its address, or 0 for None."""
    if t is None:
        return 0
    if not isinstance(t, torch.Tensor):
        _tensor(t, name)
    if (t.dtype is not dtype or t.shape != shape or t.get_device() != index
            or not t.is_contiguous()):
        _wrong(t, name, dtype, index, shape, "be contiguous")
    return t.data_ptr()


def _layout(x, name, offsets):
    """(sequences, rows per batch entry, channels, address of offsets)."""
    _tensor(x, name)
    if x.dtype not in _TYPES:
        raise TypeError("%s must be float32, bfloat16 or float16" % name)
    if not x.is_cuda:
        raise ValueError("%s must be a CUDA tensor" % name)
    shape = x.shape
    if offsets is None:
        if len(shape) != 3:
            raise ValueError("%s must be (batch, length, channels)" % name)
        return shape[0], shape[1], shape[2], 0
    if len(shape) != 2:
        raise ValueError("%s must be (rows, channels) with offsets" % name)
    _tensor(offsets, "offsets")
    if (offsets.dtype != torch.int32 or offsets.device != x.device or offsets.dim() != 1
            or offsets.shape[0] < 1 or not offsets.is_contiguous()):
        raise ValueError("offsets must be a contiguous int32 tensor of sequences + 1 "
                         "values on %s" % x.device)
    return offsets.shape[0] - 1, shape[0], shape[1], offsets.data_ptr()


def _cache(state, slots, batch, tail, dtype, index):
    """(address, entries, address of slots) of a cache that a step advances."""
    _tensor(state, "state")
    if state.dim() != 1 + len(tail):
        raise ValueError("state must have shape (entries, %s)" % ", ".join(map(str, tail)))
    n = state.shape[0]
    ptr = _flat(state, "state", dtype, index, (n,) + tail)
    if slots is None and n < batch:
        raise ValueError("state has %d entries for %d rows" % (n, batch))
    return ptr, n, _flat(slots, "slots", torch.int32, index, (batch,))


def _wants_grad(*tensors):
    if torch.is_grad_enabled():
        for t in tensors:
            if t is not None and t.requires_grad:
                return True
    return False


def _no_grad(*tensors):
    if _wants_grad(*tensors):
        raise ValueError("the single-token calls have no gradient")


def _no_tangent(*tensors):
    """Refuses forward-mode dual tensors, whose tangents a call would drop.
    Called where a dual level is open."""
    for t in tensors:
        if isinstance(t, torch.Tensor) and _forward.unpack_dual(t).tangent is not None:
            raise ValueError("the sequence operators have no forward-mode derivative")


_raise_version = torch.autograd.graph.increment_version


def _written(t):
    """A call has written t in place: operations that saved it for their
    backward pass find its version changed (inference tensors have none)."""
    if not t.is_inference():
        _raise_version(t)


def _adjacent(t):
    return t if t.shape[-1] == 1 or t.stride(-1) == 1 else t.contiguous()


def _memory(t):
    """Where the elements of t lie, in bytes: (first, [(count - 1, stride)] of the
    dimensions that are not one run, length of a run)."""
    size = t.element_size()
    run, outer = size, []
    for n, st in sorted(zip(t.shape, t.stride()), key=lambda d: d[1]):
        if n == 1:
            continue
        if st * size == run and not outer:
            run *= n
        else:
            outer.append((n - 1, st * size))
    return t.data_ptr(), outer, run


def _hits(terms, lo, hi, tries):
    """Whether a sum of x_k c_k over terms (m_k, c_k), 0 <= x_k <= m_k, falls
    into [lo, hi]: exact, from the largest c down, for layouts that nest two or
    three tries a term.  True where it takes more tries than are left."""
    terms = [t for t in terms if t[0] and t[1]]
    if not terms:
        return lo <= 0 <= hi
    (m, c), rest = terms[0], terms[1:]
    reach = sum(n * s for n, s in rest)
    for x in range(max(0, -((reach - lo) // c)), min(m, hi // c) + 1):
        tries[0] -= 1
        if not rest or tries[0] < 0 or _hits(rest, lo - x * c, hi - x * c, tries):
            return True
    return False


def _overlap(one, two):
    """Whether two layouts share a byte."""
    (a, over_a, run_a), (b, over_b, run_b) = one, two
    top = b + sum(m * c for m, c in over_b)  # the second's runs, counted down from its last
    if top + run_b <= a or a + sum(m * c for m, c in over_a) + run_a <= b:
        return False
    steps = {}
    for m, c in over_a + over_b:
        steps[c] = steps.get(c, 0) + m
    terms = sorted(((m, c) for c, m in steps.items()), key=lambda t: -t[1])
    return _hits(terms, top - a - run_a + 1, top - a + run_b - 1, [1 << 16])


def _overlaps_itself(one):
    """Whether two elements of a layout share a byte."""
    _, outer, run = one
    outer = sorted(outer, key=lambda t: -t[1])
    for k, (m, c) in enumerate(outer):
        rest = outer[k + 1:]  # at least one step of this dimension, any of the rest
        base = c - sum(n * s for n, s in rest)
        if _hits([(m - 1, c)] + [(2 * n, s) for n, s in rest], 1 - run - base, run - 1 - base,
                 [1 << 16]):
            return True
    return False


def _span(t):
    """The first byte of t's memory, and the first beyond it."""
    first = t.data_ptr()
    if t.is_contiguous():
        return first, first + t.numel() * t.element_size()
    return first, first + t.element_size() * (
        1 + sum((n - 1) * s for n, s in zip(t.shape, t.stride())))


def _apart(out, inputs, in_place=()):
    """Refuses an output that shares memory with an input or with itself; one of
    in_place may be the output."""
    if not out.numel():
        return
    if not out.is_contiguous() and _overlaps_itself(_memory(out)):
        raise ValueError("out must not overlap itself")
    lo, hi = _span(out)
    for i, t in enumerate(in_place + inputs):
        if t is None or not t.numel():
            continue
        a, b = _span(t)
        if hi <= a or b <= lo:  # nearly always
            continue
        one, to = _memory(t), _memory(out)
        if _overlap(to, one) and not (i < len(in_place) and one == to):
            raise ValueError("out must not overlap an input")


def _workspace(name, packed, device):
    _lib()
    n = _calls[name](packed)
    if n < 0:
        raise TcuDftError(2, name)
    return torch.empty(n, dtype=torch.uint8, device=device) if n else None, n


# --------------------------------------------------------- short convolution
def _width(weight):
    _tensor(weight, "weight")
    if weight.dim() != 2 or not 1 <= weight.shape[1] <= MAX_WIDTH:
        raise ValueError("weight must be (channels, width) with 1 <= width <= %d" % MAX_WIDTH)
    return weight.shape[1]


def _conv(x, weight, bias, silu, state, offsets, out, stream):
    seqs, rows, ch, off = _layout(x, "x", offsets)
    width, dtype, index = _width(weight), x.dtype, x.get_device()
    tail = (seqs, width - 1, ch)
    px = _rows(x, "x", dtype, index, x.shape)
    pw = _flat(weight, "weight", torch.float32, index, (ch, width))
    pb = _flat(bias, "bias", torch.float32, index, (ch,))
    ps = _flat(state, "state", dtype, index, tail)
    with _On(index, stream) as st:
        y = torch.empty(x.shape, dtype=dtype, device=x.device) if out is None else out
        last = torch.empty(tail, dtype=dtype, device=x.device)
        py = _rows(y, "out", dtype, index, x.shape)
        if out is not None:
            _apart(out, (x, weight, bias, state, offsets))
        if ch:
            _call("tcu_short_conv", _CONV.pack(
                _TYPES[dtype], width, bool(silu), seqs, rows, ch, off, *px, *py, *_NO_ROWS,
                *_NO_ROWS, pw, pb, ps, 0, last.data_ptr(), 0, 0, 0, 0, 0, 0, 0), st)
        if out is not None:
            _written(out)
    return y, last


class _ShortConv(torch.autograd.Function):
    @staticmethod
    def forward(ctx, x, weight, bias, state, silu, offsets):
        ctx.save_for_backward(x, weight, bias, state, offsets)
        ctx.silu = silu
        return _conv(x, weight, bias, silu, state, offsets, None, None)

    @staticmethod
    @torch.autograd.function.once_differentiable
    def backward(ctx, dy, dlast):
        x, weight, bias, state, offsets = ctx.saved_tensors
        g = short_conv_grad(_adjacent(dy), x, weight, bias, silu=ctx.silu, state=state,
                            offsets=offsets, dlast=dlast.contiguous())
        return g.x, g.weight, g.bias, g.state, None, None


def short_conv(x, weight, bias=None, *, silu=False, state=None, offsets=None, out=None,
               stream=None):
    """Depthwise causal convolution of width <= 8 over every sequence:

        p_t = bias + sum_k weight[:, k] x_{t - (width - 1) + k}

    and y = p, or p sigmoid(p) with ``silu``.  ``state`` (sequences, width - 1,
    channels), of x's type, holds the rows before each sequence (zeros if
    None).  Returns (y, last), last being the state that a continuation takes.
    """
    if _forward._current_level >= 0:
        _no_tangent(x, weight, bias, state, out)
    if _wants_grad(x, weight, bias, state):
        if out is not None or stream is not None:
            raise ValueError("out and stream cannot be given where a gradient is asked")
        return _ShortConv.apply(x, weight, bias, state, silu, offsets)
    if _wants_grad(out):
        raise ValueError("out must not record a gradient")
    return _conv(x, weight, bias, silu, state, offsets, out, stream)


def short_conv_grad(dy, x, weight, bias=None, *, silu=False, state=None, offsets=None,
                    dlast=None, stream=None):
    """Gradients of short_conv's (y, last) under dy and dlast (zeros if None):
    ConvGrads(x, weight, bias, state), the last two None where the argument is."""
    if _forward._current_level >= 0:
        _no_tangent(dy, x, weight, bias, state, dlast)
    seqs, rows, ch, off = _layout(x, "x", offsets)
    width, dtype, index, dev = _width(weight), x.dtype, x.get_device(), x.device
    tail, f32 = (seqs, width - 1, ch), torch.float32
    px = _rows(x, "x", dtype, index, x.shape)
    pdy = _rows(dy, "dy", dtype, index, x.shape)
    pw = _flat(weight, "weight", f32, index, (ch, width))
    pb = _flat(bias, "bias", f32, index, (ch,))
    ps = _flat(state, "state", dtype, index, tail)
    pl = _flat(dlast, "dlast", dtype, index, tail)
    with _On(index, stream) as st:
        dx = torch.empty(x.shape, dtype=dtype, device=dev)
        dw = torch.empty((ch, width), dtype=f32, device=dev)
        db = torch.empty((ch,), dtype=f32, device=dev) if bias is not None else None
        ds = torch.empty(tail, dtype=dtype, device=dev) if state is not None else None

        def packed(work, size):
            return _CONV.pack(
                _TYPES[dtype], width, bool(silu), seqs, rows, ch, off, *px, *_NO_ROWS, *pdy,
                *_rows(dx, "dx", dtype, index, x.shape), pw, pb, ps, pl, 0,
                ds.data_ptr() if ds is not None else 0, dw.data_ptr(),
                db.data_ptr() if db is not None else 0, work, size, 0, 0)

        if ch:
            work, n = _workspace("tcu_short_conv_grad_workspace", packed(0, 0), dev)
            _call("tcu_short_conv_grad", packed(work.data_ptr() if n else 0, n), st)
            del work
    return ConvGrads(dx, dw, db, ds)


def short_conv_step(x, state, weight, bias=None, *, silu=False, slots=None, out=None,
                    stream=None):
    """short_conv for one more row of every sequence: x (batch, channels) to y.
    ``state`` (entries, width - 1, channels) is advanced in place, at entry
    slots[b] (int32) for row b, or entry b.  A slot outside the cache gives a
    row of zeros; no two rows may name the same one."""
    if _forward._current_level >= 0:
        _no_tangent(x, state, weight, bias, out)
    _tensor(x, "x")
    if x.dim() != 2 or x.dtype not in _TYPES or not x.is_cuda:
        raise ValueError("x must be a float32, bfloat16 or float16 CUDA tensor (batch, channels)")
    _no_grad(x, state, weight, bias, out)
    batch, ch = x.shape
    width, dtype, index = _width(weight), x.dtype, x.get_device()
    cache, entries, ps = _cache(state, slots, batch, (width - 1, ch), dtype, index)
    px = _rows(x, "x", dtype, index, x.shape)
    pw = _flat(weight, "weight", torch.float32, index, (ch, width))
    pb = _flat(bias, "bias", torch.float32, index, (ch,))
    with _On(index, stream) as st:
        y = torch.empty((batch, ch), dtype=dtype, device=x.device) if out is None else out
        py = _rows(y, "out", dtype, index, x.shape)
        if out is not None:
            _apart(out, (state, weight, bias, slots), in_place=(x,))
        if ch:
            _call("tcu_short_conv_step", _CONV.pack(
                _TYPES[dtype], width, bool(silu), batch, 1, ch, 0, px[0], px[2], 0, py[0], py[2],
                0, *_NO_ROWS, *_NO_ROWS, pw, pb, 0, 0, cache, 0, 0, 0, 0, 0, ps, entries), st)
        _written(state)
        if out is not None:
            _written(out)
    return y


# ------------------------------------------------------------ selective scan
def _grouped(t, name, x):
    """B or C as (..., groups, states)."""
    _tensor(t, name)
    lead = x.dim() - 1
    if t.dim() == lead + 1:
        return t.unsqueeze(-2)
    if t.dim() != lead + 2:
        raise ValueError("%s must be (..., groups, states) or (..., states)" % name)
    return t


def _groups(B, ch):
    groups, states = B.shape[-2:]
    if not 1 <= states <= MAX_STATES:
        raise ValueError("B must have 1 to %d states" % MAX_STATES)
    if groups < 1 or ch % groups:
        raise ValueError("the %d channels must divide into the %d groups of B" % (ch, groups))
    return groups, states


class _ScanCall:
    """The checked arguments that the scan and its gradient share."""

    def __init__(self, u, dt, A, B, C, skip, gate, dt_bias, softplus, state, offsets):
        seqs, rows, ch, off = _layout(u, "u", offsets)
        B, C = _grouped(B, "B", u), _grouped(C, "C", u)
        groups, states = _groups(B, ch)
        f32, dtype, index, shape = torch.float32, u.dtype, u.get_device(), u.shape
        bc = shape[:-1] + (groups, states)
        self.index, self.dtype, self.channels, self.tail = index, dtype, ch, (seqs, ch, states)
        self.head = (_TYPES[dtype], bool(softplus), seqs, groups, rows, ch, states, off,
                     *_rows(u, "u", dtype, index, shape), *_rows(dt, "dt", dtype, index, shape),
                     *(_rows(gate, "gate", dtype, index, shape) if gate is not None else _NO_ROWS))
        self.bc = (*_grouped_rows(B, "B", dtype, index, bc), *_grouped_rows(C, "C", dtype, index, bc))
        self.params = (_flat(A, "A", f32, index, (ch, states)),
                       _flat(skip, "skip", f32, index, (ch,)),
                       _flat(dt_bias, "dt_bias", f32, index, (ch,)),
                       _flat(state, "state", f32, index, self.tail))
        batch = shape[0] if off == 0 and offsets is None else 1
        self.marks = (batch, -(-rows // MARK), ch, states)


_NO_GRADS = _NO_ROWS * 6 + (0, 0, 0)


def _scan(u, dt, A, B, C, skip, gate, dt_bias, softplus, state, offsets, marks, out, stream):
    c = _ScanCall(u, dt, A, B, C, skip, gate, dt_bias, softplus, state, offsets)
    f32, dev = torch.float32, u.device
    with _On(c.index, stream) as st:
        y = torch.empty(u.shape, dtype=u.dtype, device=dev) if out is None else out
        last = torch.empty(c.tail, dtype=f32, device=dev)
        py = _rows(y, "out", c.dtype, c.index, u.shape)
        if out is not None:
            _apart(out, (u, dt, A, B, C, skip, gate, dt_bias, state, offsets))
        kept = torch.empty(c.marks, dtype=f32, device=dev) if marks else None

        def packed(work, size):
            return _SCAN.pack(*c.head, *py, *c.bc, *c.params, 0, last.data_ptr(), 0,
                              kept.data_ptr() if marks else 0, *_NO_GRADS, work, size, 0, 0)

        if c.channels:
            work, n = _workspace("tcu_state_scan_workspace", packed(0, 0), dev)
            _call("tcu_state_scan", packed(work.data_ptr() if n else 0, n), st)
            del work
        if out is not None:
            _written(out)
    return y, last, kept


class _StateScan(torch.autograd.Function):
    @staticmethod
    def forward(ctx, u, dt, A, B, C, skip, gate, dt_bias, state, softplus, offsets):
        y, last, marks = _scan(u, dt, A, B, C, skip, gate, dt_bias, softplus, state, offsets,
                               True, None, None)
        ctx.save_for_backward(u, dt, A, B, C, skip, gate, dt_bias, state, offsets, marks)
        ctx.softplus = softplus
        return y, last

    @staticmethod
    @torch.autograd.function.once_differentiable
    def backward(ctx, dy, dlast):
        u, dt, A, B, C, skip, gate, dt_bias, state, offsets, marks = ctx.saved_tensors
        g = state_scan_grad(_adjacent(dy), u, dt, A, B, C, marks=marks, skip=skip, gate=gate,
                            dt_bias=dt_bias, softplus=ctx.softplus, state=state,
                            offsets=offsets, dlast=dlast.contiguous())
        return g.u, g.dt, g.A, g.B, g.C, g.skip, g.gate, g.dt_bias, g.state, None, None


def state_scan(u, dt, A, B, C, *, skip=None, gate=None, dt_bias=None, softplus=False, state=None,
               offsets=None, marks=False, out=None, stream=None):
    """Selective state-space scan over every sequence:

        d_t = softplus(dt_t + dt_bias)        (without ``softplus``: the sum)
        h_t = exp(d_t A) h_{t-1} + d_t u_t B_t
        o_t = sum_n C_t[n] h_t[n] + skip u_t

    and y = o, or o gate sigmoid(gate).  u, dt, gate: rows; A: (channels,
    states), states <= 128; B, C: (..., groups, states), group g serving
    channels / groups adjacent channels, or (..., states); skip, dt_bias:
    (channels,); state: (sequences, channels, states), zeros if None.

    Returns (y, last), last being the state that a continuation takes; with
    ``marks`` also the states that state_scan_grad resumes from.
    """
    if _forward._current_level >= 0:
        _no_tangent(u, dt, A, B, C, skip, gate, dt_bias, state, out)
    if _wants_grad(u, dt, A, B, C, skip, gate, dt_bias, state):
        if out is not None or marks or stream is not None:
            raise ValueError("out, marks and stream cannot be given where a gradient is asked")
        return _StateScan.apply(u, dt, A, B, C, skip, gate, dt_bias, state, softplus, offsets)
    if _wants_grad(out):
        raise ValueError("out must not record a gradient")
    y, last, kept = _scan(u, dt, A, B, C, skip, gate, dt_bias, softplus, state, offsets, marks,
                          out, stream)
    return (y, last, kept) if marks else (y, last)


def state_scan_grad(dy, u, dt, A, B, C, *, marks, skip=None, gate=None, dt_bias=None,
                    softplus=False, state=None, offsets=None, dlast=None, stream=None):
    """Gradients of state_scan's (y, last) under dy and dlast (zeros if None),
    from the marks that state_scan kept of the same arguments: ScanGrads(u, dt,
    A, B, C, skip, gate, dt_bias, state), None where the argument is."""
    if _forward._current_level >= 0:
        _no_tangent(dy, u, dt, A, B, C, marks, skip, gate, dt_bias, state, dlast)
    c = _ScanCall(u, dt, A, B, C, skip, gate, dt_bias, softplus, state, offsets)
    f32, dev, dtype, index, shape = torch.float32, u.device, c.dtype, c.index, u.shape
    pdy = _rows(dy, "dy", dtype, index, shape)
    pm = _flat(marks, "marks", f32, index, c.marks)
    pl = _flat(dlast, "dlast", f32, index, c.tail)
    with _On(index, stream) as st:
        def like(t, kind):
            return None if t is None else torch.empty(t.shape, dtype=kind, device=dev)

        def ptr(t):
            return 0 if t is None else t.data_ptr()

        def rows(t):
            return _rows(t, "gradient", dtype, index, shape) if t is not None else _NO_ROWS

        def grouped(t):
            t = _grouped(t, "gradient", u)
            return _grouped_rows(t, "gradient", dtype, index, t.shape)

        g = ScanGrads(like(u, dtype), like(dt, dtype), like(A, f32), like(B, dtype),
                      like(C, dtype), like(skip, f32), like(gate, dtype), like(dt_bias, f32),
                      like(state, f32))
        outs = (*pdy, *rows(g.u), *rows(g.dt), *rows(g.gate), *grouped(g.B), *grouped(g.C),
                ptr(g.A), ptr(g.skip), ptr(g.dt_bias))

        def packed(work, size):
            return _SCAN.pack(*c.head, *_NO_ROWS, *c.bc, *c.params, pl, 0, ptr(g.state), pm, *outs,
                              work, size, 0, 0)

        if c.channels:
            work, n = _workspace("tcu_state_scan_grad_workspace", packed(0, 0), dev)
            _call("tcu_state_scan_grad", packed(ptr(work), n), st)
            del work
        else:  # sums over no channels
            g.B.zero_()
            g.C.zero_()
    return g


def state_scan_step(u, dt, A, B, C, state, *, skip=None, gate=None, dt_bias=None, softplus=False,
                    slots=None, out=None, stream=None):
    """state_scan for one more row of every sequence: u, dt, gate (batch,
    channels), B, C (batch, groups, states) or (batch, states), to y.
    ``state`` (entries, channels, states) is advanced in place, at entry
    slots[b] (int32) for row b, or entry b.  A slot outside the cache gives a
    row of zeros; no two rows may name the same one."""
    if _forward._current_level >= 0:
        _no_tangent(u, dt, A, B, C, state, skip, gate, dt_bias, out)
    _tensor(u, "u")
    if u.dim() != 2 or u.dtype not in _TYPES or not u.is_cuda:
        raise ValueError("u must be a float32, bfloat16 or float16 CUDA tensor (batch, channels)")
    _no_grad(u, dt, A, B, C, state, skip, gate, dt_bias, out)
    batch, ch = shape = u.shape
    B, C = _grouped(B, "B", u), _grouped(C, "C", u)
    groups, states = _groups(B, ch)
    f32, dtype, index = torch.float32, u.dtype, u.get_device()
    bc = (batch, groups, states)
    cache, entries, ps = _cache(state, slots, batch, (ch, states), f32, index)
    pu, pd = _rows(u, "u", dtype, index, shape), _rows(dt, "dt", dtype, index, shape)
    pz = _rows(gate, "gate", dtype, index, shape) if gate is not None else _NO_ROWS
    pB, pC = _grouped_rows(B, "B", dtype, index, bc), _grouped_rows(C, "C", dtype, index, bc)
    pA = _flat(A, "A", f32, index, (ch, states))
    pk = _flat(skip, "skip", f32, index, (ch,))
    pi = _flat(dt_bias, "dt_bias", f32, index, (ch,))
    with _On(index, stream) as st:
        y = torch.empty((batch, ch), dtype=dtype, device=u.device) if out is None else out
        py = _rows(y, "out", dtype, index, shape)
        if out is not None:
            _apart(out, (A, B, C, state, skip, dt_bias, slots), in_place=(u, dt, gate))
        if ch:
            _call("tcu_state_scan_step", _SCAN.pack(
                _TYPES[dtype], bool(softplus), batch, groups, 1, ch, states, 0,
                pu[0], pu[2], 0, pd[0], pd[2], 0, pz[0], pz[2], 0, py[0], py[2], 0,
                pB[0], pB[2], 0, pC[0], pC[2], 0, pA, pk, pi, 0, 0, cache, 0, 0, *_NO_GRADS,
                0, 0, ps, entries), st)
        _written(state)
        if out is not None:
            _written(out)
    return y


# --------------------------------------------------- gated linear recurrence
class _GatedCall:
    """The checked arguments that the recurrence and its gradient share."""

    def __init__(self, x, forget, admit, rate, state, offsets):
        seqs, rows, ch, off = _layout(x, "x", offsets)
        f32, dtype, index, shape = torch.float32, x.dtype, x.get_device(), x.shape
        self.index, self.dtype, self.channels, self.tail = index, dtype, ch, (seqs, ch)
        self.head = (_TYPES[dtype], seqs, rows, ch, off, *_rows(x, "x", dtype, index, shape),
                     *_rows(forget, "forget", dtype, index, shape),
                     *_rows(admit, "admit", dtype, index, shape))
        self.params = (_flat(rate, "rate", f32, index, (ch,)),
                       _flat(state, "state", f32, index, self.tail))
        batch = shape[0] if offsets is None else 1
        self.marks = (batch, -(-rows // GATED_MARK), ch)


_NO_GATED_GRADS = _NO_ROWS * 4 + (0,)


def _gated(x, forget, admit, rate, state, offsets, marks, out, stream):
    c = _GatedCall(x, forget, admit, rate, state, offsets)
    f32, dev = torch.float32, x.device
    with _On(c.index, stream) as st:
        y = torch.empty(x.shape, dtype=x.dtype, device=dev) if out is None else out
        last = torch.empty(c.tail, dtype=f32, device=dev)
        py = _rows(y, "out", c.dtype, c.index, x.shape)
        if out is not None:
            _apart(out, (x, forget, admit, rate, state, offsets))
        kept = torch.empty(c.marks, dtype=f32, device=dev) if marks else None

        def packed(work, size):
            return _GATED.pack(*c.head, *py, *c.params, 0, last.data_ptr(), 0,
                               kept.data_ptr() if marks else 0, *_NO_GATED_GRADS, work, size, 0, 0)

        if c.channels:
            work, n = None, 0
            if offsets is not None:  # only packed rows take a workspace
                work, n = _workspace("tcu_gated_scan_workspace", packed(0, 0), dev)
            _call("tcu_gated_scan", packed(work.data_ptr() if n else 0, n), st)
            del work
        if out is not None:
            _written(out)
    return y, last, kept


class _GatedScan(torch.autograd.Function):
    @staticmethod
    def forward(ctx, x, forget, admit, rate, state, offsets):
        y, last, marks = _gated(x, forget, admit, rate, state, offsets, True, None, None)
        ctx.save_for_backward(x, forget, admit, rate, state, offsets, marks)
        return y, last

    @staticmethod
    @torch.autograd.function.once_differentiable
    def backward(ctx, dy, dlast):
        x, forget, admit, rate, state, offsets, marks = ctx.saved_tensors
        g = gated_scan_grad(_adjacent(dy), x, forget, admit, rate, marks=marks, state=state,
                            offsets=offsets, dlast=dlast.contiguous())
        return g.x, g.forget, g.admit, g.rate, g.state, None


def gated_scan(x, forget, admit, rate, *, state=None, offsets=None, marks=False, out=None,
               stream=None):
    """Gated linear recurrence over every sequence, one state a channel:

        a_t = exp(-rate sigmoid(forget_t))
        h_t = a_t h_{t-1} + sqrt(1 - a_t^2) sigmoid(admit_t) x_t

    and y = h.  x, forget, admit: rows; rate: (channels,), positive; state:
    (sequences, channels), zeros if None.

    Returns (y, last), last being the state that a continuation takes; with
    ``marks`` also the states that gated_scan_grad resumes from.  Rows behind
    the last packed sequence are not written.
    """
    if _forward._current_level >= 0:
        _no_tangent(x, forget, admit, rate, state, out)
    if _wants_grad(x, forget, admit, rate, state):
        if out is not None or marks or stream is not None:
            raise ValueError("out, marks and stream cannot be given where a gradient is asked")
        return _GatedScan.apply(x, forget, admit, rate, state, offsets)
    if _wants_grad(out):
        raise ValueError("out must not record a gradient")
    y, last, kept = _gated(x, forget, admit, rate, state, offsets, marks, out, stream)
    return (y, last, kept) if marks else (y, last)


def gated_scan_grad(dy, x, forget, admit, rate, *, marks, state=None, offsets=None, dlast=None,
                    stream=None):
    """Gradients of gated_scan's (y, last) under dy and dlast (zeros if None),
    from the marks that gated_scan kept of the same arguments: GatedGrads(x,
    forget, admit, rate, state), None where the argument is.  Rows behind the
    last packed sequence get zeros."""
    if _forward._current_level >= 0:
        _no_tangent(dy, x, forget, admit, rate, marks, state, dlast)
    c = _GatedCall(x, forget, admit, rate, state, offsets)
    f32, dev, dtype, index, shape = torch.float32, x.device, c.dtype, c.index, x.shape
    pdy = _rows(dy, "dy", dtype, index, shape)
    pm = _flat(marks, "marks", f32, index, c.marks)
    pl = _flat(dlast, "dlast", f32, index, c.tail)
    with _On(index, stream) as st:
        g = GatedGrads(*(torch.empty(shape, dtype=dtype, device=dev) for _ in range(3)),
                       torch.empty(rate.shape, dtype=f32, device=dev),
                       None if state is None else torch.empty(c.tail, dtype=f32, device=dev))
        outs = [v for t in g[:3] for v in _rows(t, "gradient", dtype, index, shape)]

        def packed(work, size):
            return _GATED.pack(*c.head, *_NO_ROWS, *c.params, pl, 0,
                               0 if state is None else g.state.data_ptr(), pm, *pdy, *outs,
                               g.rate.data_ptr(), work, size, 0, 0)

        if c.channels:
            work, n = _workspace("tcu_gated_scan_grad_workspace", packed(0, 0), dev)
            _call("tcu_gated_scan_grad", packed(work.data_ptr() if n else 0, n), st)
            del work
    return g


def gated_scan_step(x, forget, admit, rate, state, *, slots=None, out=None, stream=None):
    """gated_scan for one more row of every sequence: x, forget, admit (batch,
    channels) to y.  ``state`` (entries, channels) is advanced in place, at
    entry slots[b] (int32) for row b, or entry b.  A slot outside the cache
    gives a row of zeros; no two rows may name the same one."""
    if _forward._current_level >= 0:
        _no_tangent(x, forget, admit, rate, state, out)
    _tensor(x, "x")
    if x.dim() != 2 or x.dtype not in _TYPES or not x.is_cuda:
        raise ValueError("x must be a float32, bfloat16 or float16 CUDA tensor (batch, channels)")
    _no_grad(x, forget, admit, rate, state, out)
    batch, ch = shape = x.shape
    f32, dtype, index = torch.float32, x.dtype, x.get_device()
    cache, entries, ps = _cache(state, slots, batch, (ch,), f32, index)
    px, pf = _rows(x, "x", dtype, index, shape), _rows(forget, "forget", dtype, index, shape)
    pg = _rows(admit, "admit", dtype, index, shape)
    pr = _flat(rate, "rate", f32, index, (ch,))
    with _On(index, stream) as st:
        y = torch.empty((batch, ch), dtype=dtype, device=x.device) if out is None else out
        py = _rows(y, "out", dtype, index, shape)
        if out is not None:
            _apart(out, (rate, state, slots), in_place=(x, forget, admit))
        if ch:
            _call("tcu_gated_scan_step", _GATED.pack(
                _TYPES[dtype], batch, 1, ch, 0, px[0], px[2], 0, pf[0], pf[2], 0, pg[0], pg[2], 0,
                py[0], py[2], 0, pr, 0, 0, cache, 0, 0, *_NO_GATED_GRADS, 0, 0, ps, entries), st)
        _written(state)
        if out is not None:
            _written(out)
    return y
