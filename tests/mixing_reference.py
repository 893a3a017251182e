"""The gated recurrence, the head norms with rotation and the window attention
from their definitions: in 64 bits, on the CPU, with gradients by torch's
autograd; and the comparison that their GPU tests share.  Test infrastructure
only."""
import math

import torch

# Outputs are rounded once to their type: off by at most half a step.
U = {torch.float32: 2.0 ** -24, torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11}
TYPES = [torch.float32, torch.bfloat16, torch.float16]


def close(got, want, name="", inner=2e-5, terms=None):
    """The 2-norm of the error is within u + inner of the result's, inner being
    what the arithmetic before the rounding may be off; a value may lie on the
    other side of a rounding boundary, 2 u of itself, plus 5 inner of the
    result's root mean square -- or, where the sums of the terms' sizes are
    given, u and 2e-5 of them: what rounding each term by at most u can do."""
    assert got.shape == want.shape, (name, got.shape, want.shape)
    if not want.numel():
        return
    u = U[got.dtype]
    g, w = got.detach().cpu().double(), want.detach().double()
    assert torch.isfinite(g).all(), name
    err = (g - w).abs()
    norm = w.norm()
    assert err.norm() <= (u + inner) * norm + 1e-30, (name, float(err.norm() / norm))
    rms = norm / w.numel() ** 0.5
    each = 5 * inner * rms if terms is None else (u + 2e-5) * terms.detach() + 1e-4 * rms
    over = err - (2 * u * w.abs() + each)
    # numbers below the type's normal range are off by its smallest step
    assert over.max() <= torch.finfo(got.dtype).smallest_normal * u, (name, float(over.max()), float(rms))


def randn(gen, *shape, dtype=torch.float32, scale=1.0, shift=0.0):
    return (torch.randn(*shape, generator=gen) * scale + shift).to(dtype)


def packed_lengths(total, kind):
    if kind == "one":
        return [total]
    if kind == "empties":
        return [0, 0, total // 3, 0, total - total // 3, 0]
    if kind == "singles":
        return [1] * min(total, 7) + [total - min(total, 7)]
    lengths, left, k = [], total, 1
    while left > 0:
        lengths.append(min(left, 1 + (k * 37) % 61))
        left -= lengths[-1]
        k += 1
    return lengths


def offsets_of(lengths):
    o = [0]
    for n in lengths:
        o.append(o[-1] + n)
    return torch.tensor(o, dtype=torch.int32)


def cuda(d):
    return {k: v.cuda() if isinstance(v, torch.Tensor) else v for k, v in d.items()}


def doubled(d, grad=()):
    """The inputs in 64 bits, those named as leaves that record a gradient."""
    return {k: (v.detach().double().requires_grad_(k in grad)
                if isinstance(v, torch.Tensor) and v.is_floating_point() else v)
            for k, v in d.items()}


def spans(x, offsets):
    """(sequence, rows of the sequence as an index of x's leading dimensions)."""
    if offsets is None:
        return [(b, (b, slice(0, x.shape[1]))) for b in range(x.shape[0])]
    o = offsets.tolist()
    return [(s, (slice(o[s], o[s + 1]),)) for s in range(len(o) - 1)]


def logistic(v):
    return 1 / (1 + torch.exp(-v))


def gated(x, forget, admit, rate, state=None, offsets=None):
    """(y, last); rows of no sequence are zeros."""
    log = -rate * logistic(forget)
    keep, room = torch.exp(log), torch.sqrt(-torch.expm1(2 * log))
    new = room * logistic(admit) * x
    y, last = torch.zeros_like(x), []
    for s, at in spans(x, offsets):
        h, rows = (state[s] if state is not None else x.new_zeros(x.shape[-1])), []
        for t in range(new[at].shape[0]):
            h = keep[at][t] * h + new[at][t]
            rows.append(h)
        if rows:
            y = y.index_put(tuple(torch.as_tensor(i) if isinstance(i, int) else
                                  torch.arange(i.start, i.stop) for i in at), torch.stack(rows))
        last.append(h)
    return y, torch.stack(last) if last else x.new_zeros(0, x.shape[-1])


def positions_of(x, offsets):
    """The place of each row in its sequence, zero for rows of no sequence."""
    place = torch.zeros(x.shape[:-2], dtype=torch.int64)
    for _, at in spans(x, offsets):
        place[at] = torch.arange(place[at].shape[0])
    return place


def norm_rotate(x, weight, rates, positions, eps, interleaved):
    """One of the two outputs."""
    n = rates.numel()
    v = x / torch.sqrt((x * x).mean(-1, keepdim=True) + eps)
    v = v if weight is None else v * weight
    angle = positions.double()[..., None, None] * rates
    cos, sin = torch.cos(angle), torch.sin(angle)
    first, second = (v[..., 0:2 * n:2], v[..., 1:2 * n:2]) if interleaved else (v[..., :n], v[..., n:2 * n])
    a, b = first * cos - second * sin, first * sin + second * cos
    head = torch.stack([a, b], -1).flatten(-2) if interleaved else torch.cat([a, b], -1)
    return torch.cat([head, v[..., 2 * n:]], -1)


def visible(i, j, window, sinks):
    return (j <= i) & ((i - j < window) | (j < sinks))


def attention(q, k, v, window, sinks=0, scale=None, offsets=None):
    """(y, log of the sums of exponentials (..., heads, rows)); rows of no
    sequence are zeros."""
    scale = q.shape[-1] ** -0.5 if scale is None else scale
    group = q.shape[-2] // k.shape[-2]
    ys, lses = [], []
    y = torch.zeros_like(q)
    lse = q.new_zeros(q.shape[:-1])
    for _, at in spans(q, offsets):
        qs = q[at].transpose(0, 1)
        ks, vs = (x[at].transpose(0, 1).repeat_interleave(group, 0) for x in (k, v))
        n = qs.shape[1]
        if not n:
            continue
        i = torch.arange(n)
        score = scale * qs @ ks.transpose(1, 2)
        score = score.masked_fill(~visible(i[:, None], i, window, sinks), -math.inf)
        where = tuple(torch.as_tensor(a) if isinstance(a, int) else torch.arange(a.start, a.stop)
                      for a in at)
        y = y.index_put(where, (torch.softmax(score, -1) @ vs).transpose(0, 1))
        lse = lse.index_put(where, torch.logsumexp(score, -1).T)
    return y, lse


def attention_terms(q, k, v, dy, window, sinks=0, scale=None, offsets=None):
    """For each value of the gradients the sum of the sizes of its terms that
    are rounded before they are added: ds = p (dp - delta) once, and delta =
    dy.y in each product of y, for dq and dk; p for dv."""
    scale = q.shape[-1] ** -0.5 if scale is None else scale
    group = q.shape[-2] // k.shape[-2]
    out = [torch.zeros_like(t) for t in (q, k, v)]
    for _, at in spans(q, offsets):
        n = q[at].shape[0]
        if not n:
            continue
        i = torch.arange(n)
        qs, dys = q[at].transpose(0, 1), dy[at].transpose(0, 1)
        ks, vs = (x[at].transpose(0, 1).repeat_interleave(group, 0) for x in (k, v))
        score = (scale * qs @ ks.transpose(1, 2)).masked_fill(
            ~visible(i[:, None], i, window, sinks), -math.inf)
        p = torch.softmax(score, -1)
        y = p @ vs
        dp = dys @ vs.transpose(1, 2)
        size = p * ((dp - (dys * y).sum(-1, keepdim=True)).abs()
                    + (dys * y).abs().sum(-1, keepdim=True)) * scale
        out[0][at] = (size @ ks.abs()).transpose(0, 1)
        for t, x in ((out[1], size.transpose(1, 2) @ qs.abs()), (out[2], p.transpose(1, 2) @ dys.abs())):
            t[at] = x.unflatten(0, (-1, group)).sum(1).transpose(0, 1)
    return out
