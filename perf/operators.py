"""The sequence operators of this package as measured cases.

Six calls: the short causal convolution over a prompt (``conv``), with its
gradient (``conv_train``) and for one token (``conv_step``); the selective
state-space scan over a prompt (``scan``), with its gradient
(``scan_train``) and for one token (``scan_step``).

    conv:  p_t = b + sum_k w_k x_{t-(W-1)+k},      y_t = p_t sigma(p_t)
    scan:  d_t = softplus(dt_t + bias)
           h_t = exp(d_t A) h_{t-1} + d_t u_t B_t  (per channel, N states)
           y_t = (C_t . h_t + skip u_t) g_t sigma(g_t)

Where ``own`` is false ``run`` computes them with elementary torch
operations in 32 bits (the recurrence by recursive doubling over time);
where it is true it makes the package's calls.
"""
import math

import torch

own = False

TYPES = {"bf16": torch.bfloat16, "f16": torch.float16, "f32": torch.float32}


def _case(op, name=None, *, dtype="bf16", batch, length=1, channels, states=16, groups=1,
          width=4, ragged=False, carried=False):
    c = {"op": op, "dtype": dtype, "batch": batch, "channels": channels}
    if not op.endswith("step"):
        c.update(length=length, ragged=ragged)
    if op.startswith("conv"):
        c.update(width=width)
    else:
        c.update(states=states, groups=groups)
    if not op.endswith("step"):
        c.update(carried=carried)
    if name:
        c["name"] = name
    return c


def listed():
    return [
        # one short prompt of a small model: launch latency
        _case("conv", "conv short prompt", batch=1, length=37, channels=768),
        # a full prefill batch
        _case("conv", "conv prefill", batch=8, length=4096, channels=4096, carried=True),
        # documents of unequal length packed into one row of rows, in 32 bits, odd channels
        _case("conv_train", "conv train packed f32", dtype="f32", batch=13, length=317,
              channels=1031, width=3, ragged=True, carried=True),
        # a training micro-batch
        _case("conv_train", "conv train", batch=8, length=2048, channels=4096),
        # one user's next token
        _case("conv_step", "conv token x1", batch=1, channels=2048),
        # a serving batch's next tokens
        _case("conv_step", "conv token x512", batch=512, channels=4096),
        # one long document: few channels for the card, many rows
        _case("scan", "scan long document", batch=1, length=65536, channels=1536, carried=True),
        # prompts of unequal length packed for prefill, grouped B and C
        _case("scan", "scan packed prompts", dtype="f16", batch=24, length=173, channels=2048,
              groups=4, ragged=True, carried=True),
        # a small 32-bit model, odd sizes throughout
        _case("scan_train", "scan train odd f32", dtype="f32", batch=3, length=509,
              channels=331, states=13, carried=True),
        # a training micro-batch
        _case("scan_train", "scan train", batch=8, length=2048, channels=4096),
        # one user's next token
        _case("scan_step", "scan token x1", batch=1, channels=2048),
        # a serving batch's next tokens
        _case("scan_step", "scan token x512", batch=512, channels=4096),
    ]


def _between(rng, lo, hi):
    """A whole number of [lo, hi], even over its logarithm."""
    return min(hi, max(lo, int(math.exp(rng.uniform(math.log(lo), math.log(hi + 1))))))


def draw(rng):
    most = max(_cost(c) for c in listed())
    while True:
        op = rng.choice(("conv", "conv_train", "conv_step", "scan", "scan_train", "scan_step"))
        groups = rng.choice((1, 1, 1, 2, 4, 8))
        channels = _between(rng, 64, 8192)
        if rng.random() < 0.6:
            channels = -(-channels // 64) * 64
        kind = {"dtype": rng.choice(("bf16", "bf16", "f16", "f32")),
                "carried": rng.random() < 0.5, "ragged": rng.random() < 0.4}
        if op.endswith("step"):
            c = _case(op, dtype=kind["dtype"], batch=_between(rng, 1, 512),
                      channels=-(-channels // groups) * groups, groups=groups,
                      width=rng.choice((2, 3, 4)), states=rng.choice((8, 16, 16, 32, 64)))
        elif op.startswith("conv"):
            c = _case(op, batch=_between(rng, 1, 32), length=_between(rng, 1, 8192),
                      channels=channels, width=rng.choice((2, 3, 4, 4, 4, 7)), **kind)
        else:
            c = _case(op, batch=_between(rng, 1, 32),
                      length=_between(rng, 1, 65536 if op == "scan" else 8192),
                      channels=-(-channels // groups) * groups, groups=groups,
                      states=rng.choice((4, 8, 13, 16, 16, 16, 32, 64)), **kind)
        if _cost(c) <= most and _elements(c) <= 1.7e9:
            return c


def _rows(case):
    return case["batch"] * case.get("length", 1)


def _elements(case):
    return _rows(case) * case["channels"] * case.get("states", 1)


def work(case):
    size = 4 if case["dtype"] == "f32" else 2
    rows, ch, seqs = _rows(case), case["channels"], case["batch"]
    op = case["op"]
    per = rows * ch
    if op.startswith("conv"):
        w = case["width"]
        params = 4 * ch * (w + 1)
        state = size * seqs * (w - 1) * ch
        if op == "conv_step":
            return {"bytes": 2 * size * per + 2 * state + params, "flops": per * (2 * w + 5)}
        b = 2 * size * per + state * (2 if case["carried"] else 1) + params
        f = per * (2 * w + 5)
        if op == "conv_train":  # dy read, dx written; x counted once
            b += 2 * size * per + params + (state * 2 if case["carried"] else 0)
            f += per * (4 * w + 8)
        return {"bytes": b, "flops": f}
    n, g = case["states"], case["groups"]
    params = 4 * ch * (n + 2)
    state = 4 * seqs * ch * n
    bc = 2 * size * rows * g * n
    if op == "scan_step":
        return {"bytes": 4 * size * per + bc + 2 * state + params, "flops": per * (7 * n + 12)}
    b = 4 * size * per + bc + state * (2 if case["carried"] else 1) + params
    f = per * (7 * n + 12)
    if op == "scan_train":  # dy read, the gradients of u, dt, gate, B, C written
        b += 4 * size * per + bc + params + (state * 2 if case["carried"] else 0)
        f += per * (16 * n + 24)
    return {"bytes": b, "flops": f}


def _cost(case):
    w = work(case)
    return max(w["bytes"], w["flops"] / 50)


# ------------------------------------------------------------------ inputs
def _offsets(case, gen):
    """Row offsets of the packed sequences: cuts anywhere, empty ones among them."""
    rows, seqs = _rows(case), case["batch"]
    cuts = torch.randint(0, rows + 1, (seqs - 1,), generator=gen, device="cuda")
    ends = torch.tensor([rows], device="cuda")
    return torch.cat([torch.zeros_like(ends), cuts.sort().values, ends]).to(torch.int32)


def prepare(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    t = TYPES[case["dtype"]]
    op, seqs, ch = case["op"], case["batch"], case["channels"]
    step = op.endswith("step")

    def normal(*shape, dtype=t, scale=1.0, shift=0.0):
        v = torch.randn(*shape, generator=gen, device="cuda")
        return (v * scale + shift).to(dtype)

    def uniform(lo, hi, *shape):
        return torch.rand(*shape, generator=gen, device="cuda") * (hi - lo) + lo

    ragged = case.get("ragged", False)
    lead = (seqs,) if step else (_rows(case),) if ragged else (seqs, case["length"])
    s = {"case": case, "offsets": _offsets(case, gen) if ragged else None}
    f32 = torch.float32
    if op.startswith("conv"):
        w = case["width"]
        s["x"] = normal(*lead, ch)
        s["weight"] = normal(ch, w, dtype=f32, scale=w ** -0.5)
        s["bias"] = normal(ch, dtype=f32, scale=0.1)
        state = (seqs, w - 1, ch)
        state_type = t
    else:
        n, g = case["states"], case["groups"]
        s["u"], s["dt"], s["gate"] = normal(*lead, ch), normal(*lead, ch, scale=0.5), normal(*lead, ch)
        s["B"], s["C"] = normal(*lead, g, n), normal(*lead, g, n)
        rate = torch.arange(1, n + 1, device="cuda", dtype=f32)
        s["A"] = -rate * torch.exp(normal(ch, n, dtype=f32, scale=0.1))
        s["skip"] = normal(ch, dtype=f32, scale=0.1, shift=1.0)
        first = torch.exp(uniform(math.log(1e-3), math.log(1e-1), ch))
        s["dt_bias"] = torch.log(torch.expm1(first))
        state = (seqs, ch, n)
        state_type = f32
    if step:
        # a cache with more slots than the batch, taken in any order
        s["state"] = normal(2 * seqs, *state[1:], dtype=state_type)
        s["slots"] = torch.randperm(2 * seqs, generator=gen, device="cuda")[:seqs].to(torch.int32)
        return s
    s["state"] = normal(*state, dtype=state_type) if case["carried"] else None
    if op.endswith("train"):
        s["dy"] = normal(*lead, ch)
        s["dlast"] = normal(*state, dtype=state_type) if case["carried"] else None
    return s


# ------------------------------------------------------- the package's calls
def _run_own(s):
    import paper_1908_06649_gb300 as tcu

    op = s["case"]["op"]
    if op.startswith("conv"):
        x, w, b = s["x"], s["weight"], s["bias"]
        if op == "conv_step":
            y = tcu.short_conv_step(x, s["state"], w, b, silu=True, slots=s["slots"])
            return y, s["state"]
        y, last = tcu.short_conv(x, w, b, silu=True, state=s["state"], offsets=s["offsets"])
        if op == "conv":
            return y, last
        g = tcu.short_conv_grad(s["dy"], x, w, b, silu=True, state=s["state"],
                                offsets=s["offsets"], dlast=s["dlast"])
        return y, last, g.x, g.weight, g.bias, g.state
    args = (s["u"], s["dt"], s["A"], s["B"], s["C"])
    more = {"skip": s["skip"], "gate": s["gate"], "dt_bias": s["dt_bias"], "softplus": True}
    if op == "scan_step":
        y = tcu.state_scan_step(*args, s["state"], slots=s["slots"], **more)
        return y, s["state"]
    more.update(state=s["state"], offsets=s["offsets"])
    if op == "scan":
        return tcu.state_scan(*args, **more)
    y, last, marks = tcu.state_scan(*args, marks=True, **more)
    g = tcu.state_scan_grad(s["dy"], *args, marks=marks, dlast=s["dlast"], **more)
    return y, last, g.u, g.dt, g.A, g.B, g.C, g.skip, g.gate, g.dt_bias, g.state


# ------------------------------------------------------------ the plain form
def _silu(v):
    return v * torch.sigmoid(v)


def _dsilu(v):
    s = torch.sigmoid(v)
    return s * (1 + v * (1 - s))


def _layout(s):
    """(rows, sequence of each row, first row and row count of each sequence)."""
    c = s["case"]
    rows = _rows(c)
    if s["offsets"] is not None:
        off = s["offsets"].long()
    else:
        off = torch.arange(c["batch"] + 1, device="cuda") * c["length"]
    at = torch.arange(rows, device="cuda")
    return at, torch.searchsorted(off[1:].contiguous(), at, right=True), off[:-1], off[1:] - off[:-1]


def _plain_conv(s):
    # every sequence behind width-1 rows of its own past in one padded array
    t, c = TYPES[s["case"]["dtype"]], s["case"]
    w, bias, lead = s["weight"], s["bias"], c["width"] - 1
    x = s["x"].reshape(-1, c["channels"]).float()
    at, seq, first, count = _layout(s)
    k = torch.arange(lead, device="cuda")
    past = (first + lead * torch.arange(c["batch"], device="cuda"))[:, None] + k
    here = at + (seq + 1) * lead
    ends = past + count[:, None]
    padded = x.new_zeros(x.shape[0] + c["batch"] * lead, c["channels"])
    padded[here] = x
    if s["state"] is not None:
        padded[past] = s["state"].float()
    p = bias.expand_as(x)
    for j in range(lead + 1):
        p = p + w[:, j] * padded[here - lead + j]
    y, last = _silu(p).to(t).reshape(s["x"].shape), padded[ends].to(t)
    if c["op"] == "conv":
        return y, last
    dp = s["dy"].reshape(x.shape).float() * _dsilu(p)
    d = torch.zeros_like(padded)
    if s["dlast"] is not None:
        d[ends] = s["dlast"].float()
    dw = torch.empty_like(w)
    for j in range(lead + 1):
        d[here - lead + j] += w[:, j] * dp
        dw[:, j] = (dp * padded[here - lead + j]).sum(0)
    dstate = d[past].to(t) if s["state"] is not None else None
    return y, last, d[here].to(t).reshape(s["x"].shape), dw, dp.sum(0), dstate


def _plain_conv_step(s):
    t, at = s["x"].dtype, s["slots"].long()
    rows = torch.cat([s["state"][at], s["x"][:, None]], 1)
    p = (rows.float() * s["weight"].T).sum(1) + s["bias"]
    s["state"][at] = rows[:, 1:]
    return _silu(p).to(t), s["state"]


def _doubling(a, x):
    """h_t = a_t h_{t-1} + x_t along the first axis, in place of x: after the
    pass of distance k each row holds the sum over its last 2k rows."""
    k = 1
    while k < x.shape[0]:
        x[k:] += a[k:] * x[:-k]
        a[k:] *= a[:-k].clone()
        k *= 2
    return x


def _step_size(s):
    v = s["dt"].float() + s["dt_bias"]
    return torch.clamp(v, min=0) + torch.log1p(torch.exp(-v.abs()))


def _spread(v, ch):
    """(..., groups, states) of each group to its channels."""
    return v.float().repeat_interleave(ch // v.shape[-2], dim=-2)


def _plain_scan(s):
    c, t = s["case"], s["u"].dtype
    ch, n = c["channels"], c["states"]
    # rows of the dense form lie with time first, so that one scan serves all sequences
    dense = s["offsets"] is None

    def rows(v):
        return v.transpose(0, 1) if dense else v[:, None]

    def back(v):
        return (v.transpose(0, 1) if dense else v[:, 0]).to(t)

    A = s["A"]
    d, u, z = rows(_step_size(s)), rows(s["u"].float()), rows(s["gate"].float())
    B, C = rows(s["B"].float()), rows(s["C"].float())
    g = c["groups"]
    each = (g, ch // g)

    def per_group(v):  # (.., ch, n) -> (.., g, ch/g, n)
        return v.unflatten(-2, each)

    a = torch.exp(d[..., None] * A)
    x = (per_group((d * u)[..., None].expand(*u.shape, n)) * B[..., None, :]).flatten(-3, -2)
    if dense:
        if s["state"] is not None:
            x[0] += a[0] * s["state"]
        scan_a = a.clone()
    else:
        at, seq, first, count = _layout(s)
        opens = (at == first[seq])[:, None, None, None]
        if s["state"] is not None:
            x += torch.where(opens, a * s["state"][seq][:, None], 0)
        scan_a = torch.where(opens, 0, a)
    h = _doubling(scan_a, x)
    del scan_a
    if dense:
        last = h[-1].clone()
    else:
        h0 = s["state"] if s["state"] is not None else torch.zeros_like(h[:1, 0]).expand(c["batch"], ch, n)
        end = first + count - 1
        last = torch.where((count > 0)[:, None, None], h[end.clamp(min=0), 0], h0)
    out = (per_group(h) * C[..., None, :]).sum(-1).flatten(-2) + s["skip"] * u
    y = back(out * _silu(z))
    if c["op"] == "scan":
        return y, last
    dy = rows(s["dy"].float())
    dz = dy * out * _dsilu(z)
    dout = dy * _silu(z)
    # the adjoint state: e_t = C_t dout_t + a_{t+1} e_{t+1}
    e = (per_group(dout[..., None].expand(*u.shape, n)) * C[..., None, :]).flatten(-3, -2)
    nxt = torch.zeros_like(a)
    nxt[:-1] = a[1:]
    if dense:
        if s["dlast"] is not None:
            e[-1] += s["dlast"]
    else:
        closes = (at == end[seq])[:, None, None, None]
        nxt = torch.where(closes, 0, nxt)
        if s["dlast"] is not None:
            e += torch.where(closes, s["dlast"][seq][:, None], 0)
    e = _doubling(nxt.flip(0), e.flip(0)).flip(0)
    del nxt
    before = torch.zeros_like(h)
    before[1:] = h[:-1]
    if dense:
        if s["state"] is not None:
            before[0] = s["state"]
    else:
        h0s = s["state"][seq][:, None] if s["state"] is not None else 0
        before = torch.where(opens, h0s, before)
    dC = (per_group(h) * dout.unflatten(-1, each)[..., None]).sum(-2)
    dB = (per_group(e) * (d * u).unflatten(-1, each)[..., None]).sum(-2)
    dx = (per_group(e) * B[..., None, :]).sum(-1).flatten(-2)
    dstate = None
    if s["state"] is not None:
        if dense:
            dstate = a[0] * e[0]
        else:
            dstate = torch.where((count > 0)[:, None, None],
                                 (a * e)[first.clamp(max=a.shape[0] - 1), 0],
                                 s["dlast"] if s["dlast"] is not None else 0)
    a.mul_(e).mul_(before)
    dd = (a * A).sum(-1) + dx * u
    dA = (a * d[..., None]).sum((0, 1))
    v = rows(s["dt"].float()) + s["dt_bias"]
    ddt = dd * torch.sigmoid(v)
    du = dx * d + dout * s["skip"]
    dskip = (dout * u).sum((0, 1))
    return (y, last, back(du), back(ddt), dA, back(dB), back(dC), dskip, back(dz),
            ddt.sum((0, 1)), dstate)


def _plain_scan_step(s):
    at, ch = s["slots"].long(), s["case"]["channels"]
    d, u = _step_size(s), s["u"].float()
    h = torch.exp(d[..., None] * s["A"]) * s["state"][at] + (d * u)[..., None] * _spread(s["B"], ch)
    s["state"][at] = h
    out = (h * _spread(s["C"], ch)).sum(-1) + s["skip"] * u
    return (out * _silu(s["gate"].float())).to(s["u"].dtype), s["state"]


def run(state):
    if own:
        return _run_own(state)
    plain = {"conv": _plain_conv, "conv_train": _plain_conv, "conv_step": _plain_conv_step,
             "scan": _plain_scan, "scan_train": _plain_scan, "scan_step": _plain_scan_step}
    return plain[state["case"]["op"]](state)


# ------------------------------------------------- the definition in 64 bits
def _sequences(s):
    c = s["case"]
    if s["offsets"] is None:
        return [(i * c["length"], (i + 1) * c["length"]) for i in range(c["batch"])]
    o = s["offsets"].tolist()
    return list(zip(o[:-1], o[1:]))


def _exact_conv(s):
    c = s["case"]
    ch, lead = c["channels"], c["width"] - 1
    train = c["op"] == "conv_train"
    x = s["x"].reshape(-1, ch).double().requires_grad_(train)
    w, b = (s[k].double().requires_grad_(train) for k in ("weight", "bias"))
    h0 = s["state"].double().requires_grad_(train) if s["state"] is not None else None
    ys, lasts = [], []
    for i, (lo, hi) in enumerate(_sequences(s)):
        past = h0[i] if h0 is not None else x.new_zeros(lead, ch)
        long = torch.cat([past, x[lo:hi]])
        lasts.append(long[long.shape[0] - lead:])
        p = (long.unfold(0, lead + 1, 1) * w).sum(-1) + b
        ys.append(p / (1 + torch.exp(-p)))
    y, last = torch.cat(ys).reshape(s["x"].shape), torch.stack(lasts)
    if not train:
        return y, last
    outs, grads = [y], [s["dy"].double()]
    if s["dlast"] is not None:
        outs.append(last)
        grads.append(s["dlast"].double())
    leaves = [x, w, b] + ([h0] if h0 is not None else [])
    g = torch.autograd.grad(outs, leaves, grads)
    return (y.detach(), last.detach(), g[0].reshape(s["x"].shape), g[1], g[2],
            g[3] if h0 is not None else None)


def _exact_conv_step(s):
    at = s["slots"].long()
    rows = torch.cat([s["state"][at], s["x"][:, None]], 1).double()
    p = torch.einsum("bkc,ck->bc", rows, s["weight"].double()) + s["bias"].double()
    state = s["state"].double()
    state[at] = rows[:, 1:]
    return p / (1 + torch.exp(-p)), state


def _exact_scan(s):
    """Row after row, all dense sequences at once or the packed rows in one
    run whose state changes hands where a sequence opens."""
    c = s["case"]
    train = c["op"] == "scan_train"
    ch, n = c["channels"], c["states"]
    dense = s["offsets"] is None
    order = (lambda v: v.double().transpose(0, 1)) if dense else (lambda v: v.double()[:, None])
    back = (lambda v: v.transpose(0, 1)) if dense else (lambda v: v[:, 0])
    u, z, raw = order(s["u"]), order(s["gate"]), order(s["dt"]) + s["dt_bias"].double()
    d = torch.where(raw > 30, raw, torch.log1p(torch.exp(raw.clamp(max=30))))
    A, skip = s["A"].double(), s["skip"].double()
    index = torch.arange(ch, device="cuda") // (ch // c["groups"])
    B, C = order(s["B"]), order(s["C"])
    per_group = lambda v: torch.stack(  # noqa: E731
        [v[..., index == g, :].sum(-2) for g in range(c["groups"])], -2)
    rows = u.shape[0]
    zero = torch.zeros(c["batch"] if dense else 1, ch, n, device="cuda", dtype=torch.float64)
    h0 = s["state"].double() if s["state"] is not None else None
    if dense:
        opens = {0: h0 if h0 is not None else zero}
        closes = {rows - 1: s["dlast"].double() if train and s["dlast"] is not None else zero}
    else:
        spans = [(i, lo, hi) for i, (lo, hi) in enumerate(_sequences(s)) if hi > lo]
        opens = {lo: h0[i:i + 1] if h0 is not None else zero for i, lo, _ in spans}
        closes = {hi - 1: s["dlast"][i:i + 1].double() if train and s["dlast"] is not None else zero
                  for i, _, hi in spans}
    size = zero.shape[0] * ch * n * 8
    block = max(1, min(rows, int(2e9 // size)))
    y_raw, states = torch.empty_like(u), []
    h, ends = zero, {}
    for lo in range(0, rows, block):
        hi = min(rows, lo + block)
        a = torch.exp(d[lo:hi, ..., None] * A)
        hs = (d * u)[lo:hi, ..., None] * B[lo:hi][..., index, :]
        for t in range(lo, hi):
            h = opens.get(t, h)
            h = torch.addcmul(hs[t - lo], a[t - lo], h, out=hs[t - lo])
            if t in closes:
                ends[t] = h.clone()
        h = h.clone()
        y_raw[lo:hi] = torch.einsum("tbcn,tbcn->tbc", hs, C[lo:hi][..., index, :])
        if train:
            states.append(hs)
    y_raw += skip * u
    sig = 1 / (1 + torch.exp(-z))
    y = back(y_raw * z * sig)
    if dense:
        last = ends[rows - 1]
    else:
        last = h0.clone() if h0 is not None else zero.repeat(c["batch"], 1, 1)
        for i, _, hi in spans:
            last[i] = ends[hi - 1][0]
    if not train:
        return y, last
    dy = order(s["dy"])
    dz = dy * y_raw * (sig + z * sig * (1 - sig))
    q = dy * z * sig
    dA, e = torch.zeros_like(A), zero
    dd, dx = torch.empty_like(u), torch.empty_like(u)
    dB, dC = torch.zeros_like(B), torch.zeros_like(C)
    begins = {}
    for lo in reversed(range(0, rows, block)):
        hi = min(rows, lo + block)
        hs = states.pop()
        es = q[lo:hi, ..., None] * C[lo:hi][..., index, :]
        # a_t e_t of the row below, carried up
        a = torch.exp(d[lo:hi, ..., None] * A)
        for t in reversed(range(lo, hi)):
            e = es[t - lo].add_(closes[t] if t in closes else e)
            e = e * a[t - lo]
            if t in opens:
                begins[t] = e
        prev = torch.empty_like(hs)
        prev[1:] = hs[:-1]
        prev[0] = states[-1][-1] if states else 0
        for t, v in opens.items():
            if lo <= t < hi:
                prev[t - lo] = v
        dC[lo:hi] = per_group(hs * q[lo:hi, ..., None])
        del hs
        dB[lo:hi] = per_group(es * (d * u)[lo:hi, ..., None])
        dx[lo:hi] = torch.einsum("tbcn,tbcn->tbc", es, B[lo:hi][..., index, :])
        es.mul_(a).mul_(prev)
        dA += torch.einsum("tbcn,tbc->cn", es, d[lo:hi])
        dd[lo:hi] = torch.einsum("tbcn,cn->tbc", es, A)
    dd += dx * u
    ddt = dd / (1 + torch.exp(-raw))
    dstate = None
    if h0 is not None:
        if dense:
            dstate = begins[0]
        else:
            dstate = s["dlast"].double().clone() if s["dlast"] is not None else zero.repeat(c["batch"], 1, 1)
            for i, lo, _ in spans:
                dstate[i] = begins[lo][0]
    return (y, last, back(dx * d + q * skip), back(ddt), dA, back(dB), back(dC),
            (q * u).sum((0, 1)), back(dz), ddt.sum((0, 1)), dstate)


def _exact_scan_step(s):
    at, c = s["slots"].long(), s["case"]
    index = torch.arange(c["channels"], device="cuda") // (c["channels"] // c["groups"])
    u, z, raw = s["u"].double(), s["gate"].double(), s["dt"].double() + s["dt_bias"].double()
    d = torch.log1p(torch.exp(raw))
    h = torch.exp(torch.einsum("bc,cn->bcn", d, s["A"].double())) * s["state"].double()[at]
    h = h + torch.einsum("bc,bcn->bcn", d * u, s["B"].double()[:, index])
    out = torch.einsum("bcn,bcn->bc", h, s["C"].double()[:, index]) + s["skip"].double() * u
    state = s["state"].double()
    state[at] = h
    return out * z / (1 + torch.exp(-z)), state


def exact(case, seed):
    s = prepare(case, seed)
    op = case["op"]
    if op.startswith("conv"):
        return _exact_conv_step(s) if op == "conv_step" else _exact_conv(s)
    return _exact_scan_step(s) if op == "scan_step" else _exact_scan(s)
