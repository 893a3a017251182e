"""The sequence operators from their definitions: row by row, in 64 bits, on
the CPU, with gradients by torch's autograd.  Test infrastructure only."""
import torch


def spans(x, offsets):
    """(sequence, batch entry, first row, end row)."""
    if offsets is None:
        return [(b, b, 0, x.shape[1]) for b in range(x.shape[0])]
    o = offsets.tolist()
    return [(s, None, o[s], o[s + 1]) for s in range(len(o) - 1)]


def _of(x, b):
    return x if b is None else x[b]


def silu(v):
    return v / (1 + torch.exp(-v))


def softplus(v):
    return torch.where(v > 30, v, torch.log1p(torch.exp(v.clamp(max=30))))


def conv(x, weight, bias=None, act=False, state=None, offsets=None):
    ch, width = weight.shape
    y = [[] for _ in range(1 if offsets is not None else x.shape[0])]
    last = []
    for s, b, lo, hi in spans(x, offsets):
        past = state[s] if state is not None else x.new_zeros(width - 1, ch)
        rows = torch.cat([past, _of(x, b)[lo:hi]])
        last.append(rows[hi - lo:])
        for t in range(hi - lo):
            p = (rows[t:t + width] * weight.T).sum(0)
            p = p + bias if bias is not None else p
            y[b or 0].append(silu(p) if act else p)
    empty = x.new_zeros(0, ch)
    y = [torch.stack(v) if v else empty for v in y]
    last = torch.stack(last) if last else x.new_zeros(0, width - 1, ch)
    return (torch.stack(y) if offsets is None and y else (y[0] if y else x.clone())), last


def scan(u, dt, A, B, C, skip=None, gate=None, dt_bias=None, plus=False, state=None,
         offsets=None):
    ch, n = A.shape
    if B.dim() == u.dim():
        B, C = B.unsqueeze(-2), C.unsqueeze(-2)
    B, C = (v.repeat_interleave(ch // v.shape[-2], -2) for v in (B, C))
    y = [[] for _ in range(1 if offsets is not None else u.shape[0])]
    last = []
    for s, b, lo, hi in spans(u, offsets):
        h = state[s] if state is not None else u.new_zeros(ch, n)
        for t in range(lo, hi):
            d = _of(dt, b)[t]
            d = d + dt_bias if dt_bias is not None else d
            d = softplus(d) if plus else d
            ut = _of(u, b)[t]
            h = torch.exp(d[:, None] * A) * h + (d * ut)[:, None] * _of(B, b)[t]
            o = (h * _of(C, b)[t]).sum(-1)
            o = o + skip * ut if skip is not None else o
            y[b or 0].append(o * silu(_of(gate, b)[t]) if gate is not None else o)
        last.append(h)
    empty = u.new_zeros(0, ch)
    y = [torch.stack(v) if v else empty for v in y]
    last = torch.stack(last) if last else u.new_zeros(0, ch, n)
    return (torch.stack(y) if offsets is None and y else (y[0] if y else u.clone())), last
