"""Sequence operators (C ABI in include/tcu_seq.h): the short causal
convolution and the selective state-space scan, over prompts, with their
gradients, and for one token.

Rows are torch tensors of float32, bfloat16 or float16, dense -- (batch,
length, channels) -- or packed: (rows, channels) with ``offsets``, an int32
CUDA tensor of sequences + 1 row numbers from 0 to rows.  Any strides over
batch and rows are taken as they are (a slice of a wider projection needs no
copy); channels must be adjacent.  Parameters and the scan's states are
float32.  Everything runs on torch's current stream, or on ``stream``.

``short_conv`` and ``state_scan`` are differentiable: where a gradient is
asked of an argument they record themselves with autograd.  The ``_grad``
calls are what that runs; the ``_step`` calls have no gradient.
"""
from __future__ import annotations

import ctypes
from collections import namedtuple

import torch

from . import OK, TcuDftError, lib

MAX_WIDTH = 8
MAX_STATES = 128
MARK = 16  # rows from one state that the gradient resumes from to the next

SYMBOLS = (
    "tcu_short_conv", "tcu_short_conv_grad", "tcu_short_conv_grad_workspace",
    "tcu_short_conv_step", "tcu_state_scan", "tcu_state_scan_workspace",
    "tcu_state_scan_grad", "tcu_state_scan_grad_workspace",
    "tcu_state_scan_step",
)

_TYPES = {torch.float32: 0, torch.bfloat16: 1, torch.float16: 2}

ConvGrads = namedtuple("ConvGrads", "x weight bias state")
ScanGrads = namedtuple("ScanGrads", "u dt A B C skip gate dt_bias state")

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


_bound = None


def _lib():
    global _bound
    if _bound is None:
        L = lib()
        for name in SYMBOLS:
            f = getattr(L, name)
            args = ctypes.POINTER(_ConvArgs if "conv" in name else _ScanArgs)
            f.argtypes = [args] if name.endswith("workspace") else [args, _vp]
            f.restype = _i64 if name.endswith("workspace") else ctypes.c_int
        _bound = L
    return _bound


def _call(name, args, stream):
    rc = getattr(_lib(), name)(args, stream)
    if rc != OK:
        raise TcuDftError(rc, name)


class _On:
    """The device and stream of a call, current while it allocates and
    launches: memory that a call takes for itself belongs to its stream."""

    def __init__(self, device, stream):
        self.stream = stream
        self.guards = []
        if device.index != torch.cuda.current_device():
            self.guards.append(torch.cuda.device(device))
        if stream is not None:
            self.guards.append(torch.cuda.stream(stream))
        self.device = device

    def __enter__(self):
        for g in self.guards:
            g.__enter__()
        s = self.stream if self.stream is not None else torch.cuda.current_stream(self.device)
        return s.cuda_stream

    def __exit__(self, *exc):
        for g in reversed(self.guards):
            g.__exit__(*exc)


def _tensor(t, name):
    if not isinstance(t, torch.Tensor):
        raise TypeError("%s must be a torch tensor" % name)


def _rows(t, name, like, shape):
    """t as a row tensor of the type and device of `like`: (ptr, strides)."""
    _tensor(t, name)
    if t.dtype != like.dtype:
        raise TypeError("%s must be %s, not %s" % (name, like.dtype, t.dtype))
    if t.device != like.device:
        raise ValueError("%s must be on %s" % (name, like.device))
    if t.shape != shape:
        raise ValueError("%s must have shape %s, not %s" % (name, tuple(shape), tuple(t.shape)))
    st = t.stride()
    # B and C: groups and states adjacent
    if (st[-1] != 1 and shape[-1] != 1) or (
            len(shape) > like.dim() and shape[-2] > 1 and st[-2] != shape[-1]):
        raise ValueError("the values of a row of %s must be adjacent" % name)
    if like.dim() == 3:
        return _Rows(t.data_ptr(), st[0], st[1])
    return _Rows(t.data_ptr(), 0, st[0])


def _flat(t, name, dtype, device, shape):
    """t as a contiguous array, or None: its address."""
    if t is None:
        return None
    _tensor(t, name)
    if t.dtype != dtype:
        raise TypeError("%s must be %s, not %s" % (name, dtype, t.dtype))
    if t.device != device or not t.is_contiguous() or t.shape != shape:
        raise ValueError("%s must be contiguous, of shape %s, on %s"
                         % (name, tuple(shape), device))
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
        return shape[0], shape[1], shape[2], None
    if len(shape) != 2:
        raise ValueError("%s must be (rows, channels) with offsets" % name)
    _tensor(offsets, "offsets")
    if (offsets.dtype != torch.int32 or offsets.device != x.device or offsets.dim() != 1
            or offsets.shape[0] < 1 or not offsets.is_contiguous()):
        raise ValueError("offsets must be a contiguous int32 tensor of sequences + 1 "
                         "values on %s" % x.device)
    return offsets.shape[0] - 1, shape[0], shape[1], offsets.data_ptr()


def _slots(slots, batch, device):
    if slots is None:
        return None
    return _flat(slots, "slots", torch.int32, device, (batch,))


def _cache(state, slots, batch, tail, dtype, device):
    """The address and entry count of a cache that a step advances."""
    _tensor(state, "state")
    if state.dim() != 1 + len(tail):
        raise ValueError("state must have shape (entries, %s)" % ", ".join(map(str, tail)))
    n = state.shape[0]
    ptr = _flat(state, "state", dtype, device, (n,) + tail)
    if slots is None and n < batch:
        raise ValueError("state has %d entries for %d rows" % (n, batch))
    return ptr, n


def _wants_grad(*tensors):
    return torch.is_grad_enabled() and any(t is not None and t.requires_grad for t in tensors)


def _no_grad(*tensors):
    if _wants_grad(*tensors):
        raise ValueError("the single-token calls have no gradient")


# --------------------------------------------------------- short convolution
def _conv_args(x, weight, bias, silu, state, offsets):
    seqs, rows, ch, off = _layout(x, "x", offsets)
    _tensor(weight, "weight")
    if weight.dim() != 2 or not 1 <= weight.shape[1] <= MAX_WIDTH:
        raise ValueError("weight must be (channels, width) with 1 <= width <= %d" % MAX_WIDTH)
    width, f32, dev = weight.shape[1], torch.float32, x.device
    a = _ConvArgs(type=_TYPES[x.dtype], width=width, silu=bool(silu), sequences=seqs,
                  rows=rows, channels=ch, offsets=off, x=_rows(x, "x", x, x.shape),
                  weight=_flat(weight, "weight", f32, dev, (ch, width)),
                  bias=_flat(bias, "bias", f32, dev, (ch,)),
                  state=_flat(state, "state", x.dtype, dev, (seqs, width - 1, ch)))
    return a, (seqs, width - 1, ch)


def _conv(x, weight, bias, silu, state, offsets, out, stream):
    a, tail = _conv_args(x, weight, bias, silu, state, offsets)
    with _On(x.device, stream) as st:
        y = torch.empty(x.shape, dtype=x.dtype, device=x.device) if out is None else out
        last = torch.empty(tail, dtype=x.dtype, device=x.device)
        a.y = _rows(y, "out", x, x.shape)
        a.last = last.data_ptr()
        if a.channels:
            _call("tcu_short_conv", a, st)
    return y, last


class _ShortConv(torch.autograd.Function):
    @staticmethod
    def forward(ctx, x, weight, bias, state, silu, offsets, stream):
        ctx.save_for_backward(x, weight, bias, state, offsets)
        ctx.silu, ctx.stream = silu, stream
        return _conv(x, weight, bias, silu, state, offsets, None, stream)

    @staticmethod
    @torch.autograd.function.once_differentiable
    def backward(ctx, dy, dlast):
        x, weight, bias, state, offsets = ctx.saved_tensors
        g = short_conv_grad(_adjacent(dy), x, weight, bias, silu=ctx.silu, state=state,
                            offsets=offsets, dlast=dlast.contiguous(), stream=ctx.stream)
        return g.x, g.weight, g.bias, g.state, None, None, None


def _adjacent(t):
    return t if t.shape[-1] == 1 or t.stride(-1) == 1 else t.contiguous()


def short_conv(x, weight, bias=None, *, silu=False, state=None, offsets=None, out=None,
               stream=None):
    """Depthwise causal convolution of width <= 8 over every sequence:

        p_t = bias + sum_k weight[:, k] x_{t - (width - 1) + k}

    and y = p, or p sigmoid(p) with ``silu``.  ``state`` (sequences, width - 1,
    channels), of x's type, holds the rows before each sequence (zeros if
    None).  Returns (y, last), last being the state that a continuation takes.
    """
    if _wants_grad(x, weight, bias, state):
        if out is not None:
            raise ValueError("out cannot be given where a gradient is asked")
        return _ShortConv.apply(x, weight, bias, state, silu, offsets, stream)
    return _conv(x, weight, bias, silu, state, offsets, out, stream)


def short_conv_grad(dy, x, weight, bias=None, *, silu=False, state=None, offsets=None,
                    dlast=None, stream=None):
    """Gradients of short_conv's (y, last) under dy and dlast (zeros if None):
    ConvGrads(x, weight, bias, state), the last two None where the argument is."""
    a, tail = _conv_args(x, weight, bias, silu, state, offsets)
    f32, dev = torch.float32, x.device
    with _On(dev, stream) as st:
        dx = torch.empty(x.shape, dtype=x.dtype, device=dev)
        dw = torch.empty(weight.shape, dtype=f32, device=dev)
        db = torch.empty(bias.shape, dtype=f32, device=dev) if bias is not None else None
        ds = torch.empty(tail, dtype=x.dtype, device=dev) if state is not None else None
        a.dy, a.dx = _rows(dy, "dy", x, x.shape), _rows(dx, "dx", x, x.shape)
        a.dlast = _flat(dlast, "dlast", x.dtype, dev, tail)
        a.dweight = dw.data_ptr()
        a.dbias = db.data_ptr() if db is not None else None
        a.dstate = ds.data_ptr() if ds is not None else None
        if a.channels:
            work = _workspace("tcu_short_conv_grad_workspace", a, dev)
            _call("tcu_short_conv_grad", a, st)
            del work
    return ConvGrads(dx, dw, db, ds)


def _workspace(name, a, device):
    n = getattr(_lib(), name)(a)
    if n < 0:
        raise TcuDftError(2, name)
    w = torch.empty(n, dtype=torch.uint8, device=device)
    a.workspace, a.workspace_bytes = w.data_ptr(), n
    return w


def short_conv_step(x, state, weight, bias=None, *, silu=False, slots=None, out=None,
                    stream=None):
    """short_conv for one more row of every sequence: x (batch, channels) to y.
    ``state`` (entries, width - 1, channels) is advanced in place, at entry
    slots[b] (int32) for row b, or entry b.  A slot outside the cache gives a
    row of zeros; no two rows may name the same one."""
    _no_grad(x, weight, bias)
    _tensor(x, "x")
    _tensor(weight, "weight")
    if x.dim() != 2 or x.dtype not in _TYPES or not x.is_cuda:
        raise ValueError("x must be a float32, bfloat16 or float16 CUDA tensor (batch, channels)")
    if weight.dim() != 2 or not 1 <= weight.shape[1] <= MAX_WIDTH:
        raise ValueError("weight must be (channels, width) with 1 <= width <= %d" % MAX_WIDTH)
    batch, ch = x.shape
    width, f32, dev = weight.shape[1], torch.float32, x.device
    ptr, entries = _cache(state, slots, batch, (width - 1, ch), x.dtype, dev)
    with _On(dev, stream) as st:
        y = torch.empty((batch, ch), dtype=x.dtype, device=dev) if out is None else out
        a = _ConvArgs(type=_TYPES[x.dtype], width=width, silu=bool(silu), sequences=batch, rows=1,
                      channels=ch, x=_step_rows(x, "x", x, x.shape),
                      y=_step_rows(y, "out", x, x.shape),
                      weight=_flat(weight, "weight", f32, dev, (ch, width)),
                      bias=_flat(bias, "bias", f32, dev, (ch,)), last=ptr,
                      slots=_slots(slots, batch, dev), num_slots=entries)
        if ch:
            _call("tcu_short_conv_step", a, st)
    return y


def _step_rows(t, name, like, shape):
    r = _rows(t, name, like, shape)
    return _Rows(r.ptr, r.row_stride, 0)


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


def _scan_args(u, dt, A, B, C, skip, gate, dt_bias, softplus, state, offsets):
    seqs, rows, ch, off = _layout(u, "u", offsets)
    B, C = _grouped(B, "B", u), _grouped(C, "C", u)
    groups, states = B.shape[-2:]
    if not 1 <= states <= MAX_STATES:
        raise ValueError("B must have 1 to %d states" % MAX_STATES)
    if groups < 1 or ch % groups:
        raise ValueError("the %d channels must divide into the %d groups of B" % (ch, groups))
    f32, dev, lead = torch.float32, u.device, tuple(u.shape[:-1])
    bc = torch.Size(lead + (groups, states))
    a = _ScanArgs(type=_TYPES[u.dtype], softplus=bool(softplus), sequences=seqs, groups=groups,
                  rows=rows, channels=ch, states=states, offsets=off,
                  u=_rows(u, "u", u, u.shape), dt=_rows(dt, "dt", u, u.shape),
                  B=_rows(B, "B", u, bc), C=_rows(C, "C", u, bc),
                  A=_flat(A, "A", f32, dev, (ch, states)),
                  skip=_flat(skip, "skip", f32, dev, (ch,)),
                  dt_bias=_flat(dt_bias, "dt_bias", f32, dev, (ch,)),
                  state=_flat(state, "state", f32, dev, (seqs, ch, states)))
    if gate is not None:
        a.gate = _rows(gate, "gate", u, u.shape)
    return a, (seqs, ch, states)


def _marks_shape(u, offsets, states):
    batch, rows = (u.shape[0], u.shape[1]) if offsets is None else (1, u.shape[0])
    return (batch, -(-rows // MARK), u.shape[-1], states)


def _scan(u, dt, A, B, C, skip, gate, dt_bias, softplus, state, offsets, marks, out, stream):
    a, tail = _scan_args(u, dt, A, B, C, skip, gate, dt_bias, softplus, state, offsets)
    f32, dev = torch.float32, u.device
    with _On(dev, stream) as st:
        y = torch.empty(u.shape, dtype=u.dtype, device=dev) if out is None else out
        last = torch.empty(tail, dtype=f32, device=dev)
        a.y = _rows(y, "out", u, u.shape)
        a.last = last.data_ptr()
        kept = None
        if marks:
            kept = torch.empty(_marks_shape(u, offsets, tail[2]), dtype=f32, device=dev)
            a.marks = kept.data_ptr()
        if a.channels:
            work = _workspace("tcu_state_scan_workspace", a, dev)
            _call("tcu_state_scan", a, st)
            del work
    return y, last, kept


class _StateScan(torch.autograd.Function):
    @staticmethod
    def forward(ctx, u, dt, A, B, C, skip, gate, dt_bias, state, softplus, offsets, stream):
        y, last, marks = _scan(u, dt, A, B, C, skip, gate, dt_bias, softplus, state, offsets,
                               True, None, stream)
        ctx.save_for_backward(u, dt, A, B, C, skip, gate, dt_bias, state, offsets, marks)
        ctx.softplus, ctx.stream = softplus, stream
        return y, last

    @staticmethod
    @torch.autograd.function.once_differentiable
    def backward(ctx, dy, dlast):
        u, dt, A, B, C, skip, gate, dt_bias, state, offsets, marks = ctx.saved_tensors
        g = state_scan_grad(_adjacent(dy), u, dt, A, B, C, marks=marks, skip=skip, gate=gate,
                            dt_bias=dt_bias, softplus=ctx.softplus, state=state,
                            offsets=offsets, dlast=dlast.contiguous(), stream=ctx.stream)
        return g.u, g.dt, g.A, g.B, g.C, g.skip, g.gate, g.dt_bias, g.state, None, None, None


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
    if _wants_grad(u, dt, A, B, C, skip, gate, dt_bias, state):
        if out is not None or marks:
            raise ValueError("out and marks cannot be given where a gradient is asked")
        return _StateScan.apply(u, dt, A, B, C, skip, gate, dt_bias, state, softplus, offsets,
                                stream)
    y, last, kept = _scan(u, dt, A, B, C, skip, gate, dt_bias, softplus, state, offsets, marks,
                          out, stream)
    return (y, last, kept) if marks else (y, last)


def state_scan_grad(dy, u, dt, A, B, C, *, marks, skip=None, gate=None, dt_bias=None,
                    softplus=False, state=None, offsets=None, dlast=None, stream=None):
    """Gradients of state_scan's (y, last) under dy and dlast (zeros if None),
    from the marks that state_scan kept of the same arguments: ScanGrads(u, dt,
    A, B, C, skip, gate, dt_bias, state), None where the argument is."""
    a, tail = _scan_args(u, dt, A, B, C, skip, gate, dt_bias, softplus, state, offsets)
    f32, dev = torch.float32, u.device
    with _On(dev, stream) as st:
        def like(t, dtype):
            return None if t is None else torch.empty(t.shape, dtype=dtype, device=dev)

        g = ScanGrads(like(u, u.dtype), like(dt, u.dtype), like(A, f32), like(B, u.dtype),
                      like(C, u.dtype), like(skip, f32), like(gate, u.dtype),
                      like(dt_bias, f32), like(state, f32))
        a.dy = _rows(dy, "dy", u, u.shape)
        a.marks = _flat(marks, "marks", f32, dev, _marks_shape(u, offsets, tail[2]))
        a.dlast = _flat(dlast, "dlast", f32, dev, tail)
        a.du, a.ddt = _rows(g.u, "du", u, u.shape), _rows(g.dt, "ddt", u, u.shape)
        for name, t in (("dB", g.B), ("dC", g.C)):
            t = _grouped(t, name, u)
            setattr(a, name, _rows(t, name, u, t.shape))
        if gate is not None:
            a.dgate = _rows(g.gate, "dgate", u, u.shape)
        for name, t in (("dA", g.A), ("dskip", g.skip), ("ddt_bias", g.dt_bias),
                        ("dstate", g.state)):
            setattr(a, name, t.data_ptr() if t is not None else None)
        if a.channels:
            work = _workspace("tcu_state_scan_grad_workspace", a, dev)
            _call("tcu_state_scan_grad", a, st)
            del work
    return g


def state_scan_step(u, dt, A, B, C, state, *, skip=None, gate=None, dt_bias=None, softplus=False,
                    slots=None, out=None, stream=None):
    """state_scan for one more row of every sequence: u, dt, gate (batch,
    channels), B, C (batch, groups, states) or (batch, states), to y.
    ``state`` (entries, channels, states) is advanced in place, at entry
    slots[b] (int32) for row b, or entry b.  A slot outside the cache gives a
    row of zeros; no two rows may name the same one."""
    _no_grad(u, dt, A, B, C, skip, gate, dt_bias)
    _tensor(u, "u")
    if u.dim() != 2 or u.dtype not in _TYPES or not u.is_cuda:
        raise ValueError("u must be a float32, bfloat16 or float16 CUDA tensor (batch, channels)")
    batch, ch = u.shape
    B, C = _grouped(B, "B", u), _grouped(C, "C", u)
    groups, states = B.shape[-2:]
    if not 1 <= states <= MAX_STATES:
        raise ValueError("B must have 1 to %d states" % MAX_STATES)
    if groups < 1 or ch % groups:
        raise ValueError("the %d channels must divide into the %d groups of B" % (ch, groups))
    f32, dev = torch.float32, u.device
    bc = torch.Size((batch, groups, states))
    ptr, entries = _cache(state, slots, batch, (ch, states), f32, dev)
    with _On(dev, stream) as st:
        y = torch.empty((batch, ch), dtype=u.dtype, device=dev) if out is None else out
        a = _ScanArgs(type=_TYPES[u.dtype], softplus=bool(softplus), sequences=batch,
                      groups=groups, rows=1, channels=ch, states=states,
                      u=_step_rows(u, "u", u, u.shape), dt=_step_rows(dt, "dt", u, u.shape),
                      y=_step_rows(y, "out", u, u.shape), B=_step_rows(B, "B", u, bc),
                      C=_step_rows(C, "C", u, bc), A=_flat(A, "A", f32, dev, (ch, states)),
                      skip=_flat(skip, "skip", f32, dev, (ch,)),
                      dt_bias=_flat(dt_bias, "dt_bias", f32, dev, (ch,)), last=ptr,
                      slots=_slots(slots, batch, dev), num_slots=entries)
        if gate is not None:
            a.gate = _step_rows(gate, "gate", u, u.shape)
        if ch:
            _call("tcu_state_scan_step", a, st)
    return y
