"""The operators of recurrence and local attention as measured cases.

    gated    a_t = exp(-rate s(forget_t))                       (per channel)
             h_t = a_t h_{t-1} + sqrt(1 - a_t^2) s(admit_t) x_t,  y_t = h_t
    rotate   n = x / sqrt(mean(x^2) + eps) * weight             (per head of q and k)
             pairs (n_p, n_{p + r}) turned by the angle position * rates_p
    attend   y_i = sum_j p_ij v_j,  p = softmax over the visible j of scale q_i.k_j
             j visible to i: j <= i and (i - j < window or j < sinks)

s is the logistic function.  Each over prompts, with its gradient (``train``)
and for single tokens (``token``; attention and recurrence from caches).

Where ``own`` is false ``run`` computes them with elementary torch operations
in 32 bits (angles in 64; the recurrence by recursive doubling over time,
attention by blocks of a window's rows); where it is true it makes the
package's calls.
"""
import math

import torch

own = False

TYPES = {"bf16": torch.bfloat16, "f16": torch.float16, "f32": torch.float32}
EPS = 1e-6


def _gated(op, name=None, *, dtype="bf16", batch, channels, length=1, ragged=False, carried=False):
    c = {"op": "gated_" + op, "dtype": dtype, "batch": batch, "channels": channels}
    if op != "token":
        c.update(length=length, ragged=ragged, carried=carried)
    return dict(c, name=name) if name else c


def _rotate(op, name=None, *, dtype="bf16", batch, heads, kv_heads, dim, turned, length=1,
            ragged=False, far=0, interleaved=False):
    c = {"op": "rotate_" + op, "dtype": dtype, "batch": batch, "heads": heads,
         "kv_heads": kv_heads, "dim": dim, "turned": turned, "far": far,
         "interleaved": interleaved}
    if op != "token":
        c.update(length=length, ragged=ragged)
    return dict(c, name=name) if name else c


def _attend(op, name=None, *, dtype="bf16", batch, heads, kv_heads, dim, window, sinks, length=1,
            ragged=False):
    c = {"op": "attend_" + op, "dtype": dtype, "batch": batch, "heads": heads,
         "kv_heads": kv_heads, "dim": dim, "window": window, "sinks": sinks}
    if op != "token":
        c.update(length=length, ragged=ragged)
    return dict(c, name=name) if name else c


def listed():
    return [
        # a serving batch's next tokens
        _gated("token", "gated token x128", batch=128, channels=4096),
        # one long document: few channels for the card, many rows
        _gated("prompt", "gated long document", batch=1, length=65536, channels=1536, carried=True),
        # documents of unequal length packed into one row of rows, in 32 bits, odd channels
        _gated("train", "gated train packed f32", dtype="f32", batch=13, length=317, channels=1031,
               ragged=True, carried=True),
        # a training micro-batch
        _gated("train", "gated train", batch=8, length=2048, channels=4096),
        # one user's next token, far into a document: launch latency
        _rotate("token", "rotate token x1", batch=1, heads=16, kv_heads=4, dim=128, turned=128,
                far=1 << 20),
        # prompts of unequal length packed for prefill, odd heads, half of a head turned
        _rotate("prompt", "rotate packed prompts", dtype="f16", batch=24, length=173, heads=10,
                kv_heads=5, dim=80, turned=40, ragged=True, interleaved=True),
        # a training micro-batch
        _rotate("train", "rotate train", batch=8, length=2048, heads=32, kv_heads=8, dim=128,
                turned=128),
        # one user's next token: launch latency
        _attend("token", "attend token x1", batch=1, heads=16, kv_heads=4, dim=128, window=1024,
                sinks=4),
        # a serving batch's next tokens
        _attend("token", "attend token x64", batch=64, heads=32, kv_heads=8, dim=128, window=2048,
                sinks=4),
        # prefill of one long document, which leaves its cache
        _attend("prompt", "attend long document", batch=1, length=32768, heads=32, kv_heads=8,
                dim=128, window=2048, sinks=4),
        # documents of unequal length packed, odd heads, a window that ends inside tiles
        _attend("train", "attend train packed", dtype="f16", batch=13, length=317, heads=10,
                kv_heads=5, dim=80, window=200, sinks=3, ragged=True),
        # a training micro-batch
        _attend("train", "attend train", batch=4, length=2048, heads=16, kv_heads=4, dim=128,
                window=1024, sinks=4),
    ]


def _between(rng, lo, hi):
    """A whole number of [lo, hi], even over its logarithm."""
    return min(hi, max(lo, int(math.exp(rng.uniform(math.log(lo), math.log(hi + 1))))))


def draw(rng):
    most = max(_cost(c) for c in listed())
    while True:
        kind = rng.choice(("gated", "rotate", "attend"))
        op = rng.choice(("prompt", "train", "token"))
        dtype = rng.choice(("bf16", "bf16", "f16") if kind == "attend"
                           else ("bf16", "bf16", "f16", "f32"))
        more = {"dtype": dtype, "batch": _between(rng, 1, 256 if op == "token" else 32)}
        if op != "token":
            more.update(length=_between(rng, 1, 65536 if kind == "gated" else 16384),
                        ragged=rng.random() < 0.4)
        if kind == "gated":
            channels = _between(rng, 64, 8192)
            if rng.random() < 0.6:
                channels = -(-channels // 64) * 64
            if op != "token":
                more["carried"] = rng.random() < 0.5
            c = _gated(op, channels=channels, **more)
        else:
            kv, group = rng.choice((1, 2, 3, 4, 5, 8)), rng.choice((1, 2, 3, 4, 4, 7, 8))
            more.update(heads=kv * group, kv_heads=kv)
            if kind == "rotate":
                dim = rng.choice((32, 64, 64, 80, 96, 128, 128, 128, 256))
                c = _rotate(op, dim=dim, turned=rng.choice((dim, dim, dim // 2)),
                            far=rng.choice((0, 0, _between(rng, 1, 1 << 20))),
                            interleaved=rng.random() < 0.3, **more)
            else:
                c = _attend(op, dim=rng.choice((32, 64, 64, 80, 96, 128, 128, 128)),
                            window=_between(rng, 1, 4096), sinks=rng.choice((0, 1, 4, 4, 16)),
                            **more)
        if _cost(c) <= most and _fits(c):
            return c


def _rows(case):
    return case["batch"] * case.get("length", 1)


def _fits(case):
    """Whether the plain form's arrays stay within some 20 GB each."""
    rows = _rows(case)
    if case["op"].startswith("gated"):
        return rows * case["channels"] <= 1.4e8
    if case["op"].startswith("rotate"):
        return rows * case["heads"] * case["dim"] <= 4e8
    kv = case["kv_heads"] * case["dim"]
    if case["op"] == "attend_token":
        return 2 * rows * (case["window"] + case["sinks"]) * kv <= 4e8
    return (rows * 2 * min(case["window"], rows) * case["heads"] <= 4.4e9
            and rows * case["sinks"] * kv <= 1.1e9
            and 2 * case["batch"] * (case["window"] + case["sinks"]) * kv <= 4e8)


def _pairs(case):
    """Visible pairs of one sequence and head, of equal sequences."""
    n, w, s = case["length"], case["window"], case["sinks"]
    m = min(n, w)
    pairs = m * (m + 1) // 2 + (n - m) * w
    beyond = max(0, n - w)  # rows that see sinks outside their window
    t = min(beyond, s)
    return pairs + t * (t + 1) // 2 + (beyond - t) * s


def work(case):
    op, rows = case["op"], _rows(case)
    size = 4 if case["dtype"] == "f32" else 2
    if op.startswith("gated"):
        per = rows * case["channels"]
        state = 4 * case["batch"] * case["channels"]
        params = 4 * case["channels"]
        if op == "gated_token":
            return {"bytes": 4 * size * per + 2 * state + params, "flops": 20 * per}
        b = 4 * size * per + state * (2 if case["carried"] else 1) + params
        if op == "gated_prompt":
            return {"bytes": b, "flops": 20 * per}
        # dy read, the gradients of x and both gates written; x and the gates counted once
        b += 4 * size * per + params + (2 * state if case["carried"] else 0)
        return {"bytes": b, "flops": 60 * per}
    d, h, kv = case["dim"], case["heads"], case["kv_heads"]
    if op.startswith("rotate"):
        per, params = rows * (h + kv) * d, 8 * d + 2 * case["turned"]
        if op != "rotate_train":
            return {"bytes": 2 * size * per + 4 * rows + params, "flops": 8 * per}
        return {"bytes": 4 * size * per + 4 * rows + params + 8 * d, "flops": 30 * per}
    qs, ks = size * rows * h * d, size * rows * kv * d
    if op == "attend_token":
        seen = case["window"] + case["sinks"]
        return {"bytes": 2 * qs + 2 * ks + 2 * ks * seen + 8 * rows, "flops": 4 * d * rows * h * seen}
    f = 4 * d * h * case["batch"] * _pairs(case)
    if op == "attend_prompt":
        entry = min(case["length"], case["window"] + case["sinks"])
        return {"bytes": 2 * qs + 2 * ks + 2 * size * case["batch"] * entry * kv * d, "flops": f}
    # q, k, v, dy read; y and three gradients written
    return {"bytes": 4 * qs + 4 * ks, "flops": 7 * f // 2}


def _cost(case):
    w = work(case)
    return max(w["bytes"], w["flops"] / 200)


# ------------------------------------------------------------------ inputs
def _offsets(case, gen):
    """Row offsets of the packed sequences: cuts anywhere, empty ones among them."""
    rows, seqs = _rows(case), case["batch"]
    cuts = torch.randint(0, rows + 1, (seqs - 1,), generator=gen, device="cuda")
    ends = torch.tensor([rows], device="cuda")
    return torch.cat([torch.zeros_like(ends), cuts.sort().values, ends]).to(torch.int32)


def prepare(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    t, op, seqs = TYPES[case["dtype"]], case["op"], case["batch"]
    token, train = op.endswith("token"), op.endswith("train")

    def normal(*shape, dtype=t, scale=1.0, shift=0.0):
        v = torch.randn(*shape, generator=gen, device="cuda")
        return (v * scale + shift).to(dtype)

    def slots(entries):
        # a cache with more slots than the batch, taken in any order
        return torch.randperm(entries, generator=gen, device="cuda")[:seqs].to(torch.int32)

    ragged = case.get("ragged", False)
    lead = (seqs,) if token else (_rows(case),) if ragged else (seqs, case["length"])
    s = {"case": case, "offsets": _offsets(case, gen) if ragged else None}
    f32 = torch.float32
    if op.startswith("gated"):
        ch = case["channels"]
        s["x"], s["forget"], s["admit"] = normal(*lead, ch), normal(*lead, ch), normal(*lead, ch)
        # decays a^(1/2) between 0.9 and 0.999 at a gate that is half open
        keep = torch.rand(ch, generator=gen, device="cuda") * 0.099 + 0.9
        s["rate"] = -2 * torch.log(keep)
        if token:
            s["state"], s["slots"] = normal(2 * seqs, ch, dtype=f32), slots(2 * seqs)
            return s
        s["state"] = normal(seqs, ch, dtype=f32) if case["carried"] else None
        if train:
            s["dy"] = normal(*lead, ch)
            s["dlast"] = normal(seqs, ch, dtype=f32) if case["carried"] else None
        return s
    h, kv, d = case["heads"], case["kv_heads"], case["dim"]
    if op.startswith("rotate"):
        # queries and keys lie side by side, as a projection leaves them
        both = normal(*lead, h + kv, d, scale=2.0)
        s["q"], s["k"] = both[..., :h, :], both[..., h:, :]
        s["q_weight"] = normal(d, dtype=f32, scale=0.1, shift=1.0)
        s["k_weight"] = normal(d, dtype=f32, scale=0.1, shift=1.0)
        n = case["turned"] // 2
        s["rates"] = 10000.0 ** (-torch.arange(n, device="cuda", dtype=f32) / n)
        s["positions"] = None
        if token:
            s["positions"] = torch.randint(0, case["far"] + 1, lead, generator=gen,
                                           device="cuda", dtype=torch.int32)
        elif case["far"] and not ragged:
            # chunks of longer documents
            first = torch.randint(0, case["far"] + 1, (seqs, 1), generator=gen, device="cuda")
            s["positions"] = (first + torch.arange(case["length"], device="cuda")).to(torch.int32)
        if train:
            s["dq"], s["dk"] = normal(*lead, h, d), normal(*lead, kv, d)
        return s
    s["q"], s["k"], s["v"] = normal(*lead, h, d), normal(*lead, kv, d), normal(*lead, kv, d)
    seen = case["window"] + case["sinks"]
    if token:
        s["cache"] = normal(2, 2 * seqs, seen, kv, d)
        s["slots"] = slots(2 * seqs)
        # most sequences are longer than their window
        s["positions"] = torch.randint(seen // 2, 4 * seen, lead, generator=gen, device="cuda",
                                       dtype=torch.int32)
    elif train:
        s["dy"] = normal(*lead, h, d)
    else:
        s["cache"] = torch.zeros(2, 2 * seqs, seen, kv, d, dtype=t, device="cuda")
        s["slots"] = slots(2 * seqs)
    return s


# ------------------------------------------------------- the package's calls
def _run_own(s):
    import paper_1908_06649_gb300 as tcu

    op = s["case"]["op"]
    if op.startswith("gated"):
        args = (s["x"], s["forget"], s["admit"], s["rate"])
        if op == "gated_token":
            return tcu.gated_scan_step(*args, s["state"], slots=s["slots"]), s["state"]
        more = {"state": s["state"], "offsets": s["offsets"]}
        if op == "gated_prompt":
            return tcu.gated_scan(*args, **more)
        y, last, marks = tcu.gated_scan(*args, marks=True, **more)
        g = tcu.gated_scan_grad(s["dy"], *args, marks=marks, dlast=s["dlast"], **more)
        return y, last, g.x, g.forget, g.admit, g.rate, g.state
    if op.startswith("rotate"):
        args = (s["q"], s["k"], s["rates"])
        more = {"q_weight": s["q_weight"], "k_weight": s["k_weight"], "eps": EPS,
                "positions": s["positions"], "offsets": s["offsets"],
                "interleaved": s["case"]["interleaved"]}
        q, k = tcu.norm_rotate(*args, **more)
        if op != "rotate_train":
            return q, k
        g = tcu.norm_rotate_grad(s["dq"], s["dk"], *args, **more)
        return q, k, g.q, g.k, g.q_weight, g.k_weight
    qkv = (s["q"], s["k"], s["v"])
    more = {"window": s["case"]["window"], "sinks": s["case"]["sinks"]}
    if op == "attend_token":
        y = tcu.window_attention_step(*qkv, *s["cache"].unbind(0), s["positions"],
                                      slots=s["slots"], **more)
        return y, s["cache"]
    more["offsets"] = s["offsets"]
    if op == "attend_prompt":
        y = tcu.window_attention(*qkv, **more)
        tcu.window_cache(s["k"], s["v"], *s["cache"].unbind(0), slots=s["slots"], **more)
        return y, s["cache"]
    y, lse = tcu.window_attention(*qkv, lse=True, **more)
    g = tcu.window_attention_grad(s["dy"], *qkv, y, lse, **more)
    return y, g.q, g.k, g.v


# ------------------------------------------------------------ the plain form
def _layout(s):
    """(rows, sequence of each row, first row and row count of each sequence)."""
    c = s["case"]
    rows = _rows(c)
    if s["offsets"] is not None:
        off = s["offsets"].long()
    else:
        off = torch.arange(c["batch"] + 1, device="cuda") * c.get("length", 1)
    at = torch.arange(rows, device="cuda")
    return at, torch.searchsorted(off[1:].contiguous(), at, right=True), off[:-1], off[1:] - off[:-1]


def _doubling(a, x):
    """h_t = a_t h_{t-1} + x_t along the first axis, in place of x: after the
    pass of distance k each row holds the sum over its last 2k rows."""
    k = 1
    while k < x.shape[0]:
        x[k:] += a[k:] * x[:-k]
        a[k:] *= a[:-k].clone()
        k *= 2
    return x


def _plain_gated(s):
    c, t = s["case"], s["x"].dtype
    rate = s["rate"]
    if c["op"] == "gated_token":
        at = s["slots"].long()
        log = -rate * torch.sigmoid(s["forget"].float())
        new = torch.sqrt(-torch.expm1(2 * log)) * torch.sigmoid(s["admit"].float()) * s["x"].float()
        h = torch.exp(log) * s["state"][at] + new
        s["state"][at] = h
        return h.to(t), s["state"]
    # rows of the dense form lie with time first, so that one scan serves all sequences
    dense = s["offsets"] is None

    def rows(v):
        return v.float().transpose(0, 1) if dense else v.float()[:, None]

    def back(v):
        return (v.transpose(0, 1) if dense else v[:, 0]).to(t)

    x, open_f, open_a = rows(s["x"]), torch.sigmoid(rows(s["forget"])), torch.sigmoid(rows(s["admit"]))
    log = -rate * open_f
    # decays near one in 64 bits: a recurrence of many rows multiplies their mean error
    a = torch.exp(log.double()).float()
    root = torch.sqrt(-torch.expm1(2 * log))
    new = root * open_a * x
    if dense:
        if s["state"] is not None:
            new[0] += a[0] * s["state"]
        h = _doubling(a.clone(), new)
        last = h[-1].clone()
    else:
        at, seq, first, count = _layout(s)
        opens = (at == first[seq])[:, None, None]
        if s["state"] is not None:
            new += torch.where(opens, a * s["state"][seq][:, None], 0)
        h = _doubling(torch.where(opens, 0, a), new)
        end = first + count - 1
        h0 = s["state"] if s["state"] is not None else torch.zeros_like(h[:1, 0]).expand(c["batch"], -1)
        last = torch.where((count > 0)[:, None], h[end.clamp(min=0), 0], h0)
    y = back(h)
    if c["op"] == "gated_prompt":
        return y, last
    # the adjoint: e_t = dy_t + a_{t+1} e_{t+1}
    e = rows(s["dy"]).clone()
    nxt, before = torch.zeros_like(a), torch.zeros_like(a)
    nxt[:-1], before[1:] = a[1:], h[:-1]
    if dense:
        if s["dlast"] is not None:
            e[-1] += s["dlast"]
        if s["state"] is not None:
            before[0] = s["state"]
    else:
        closes = (at == end[seq])[:, None, None]
        nxt = torch.where(closes, 0, nxt)
        if s["dlast"] is not None:
            e += torch.where(closes, s["dlast"][seq][:, None], 0)
        before = torch.where(opens, s["state"][seq][:, None] if s["state"] is not None else 0, before)
    e = _doubling(nxt.flip(0), e.flip(0)).flip(0)
    dx, da = e * root * open_a, e * root * x * open_a * (1 - open_a)
    # d log a: through a and through the root of 1 - a^2
    dlog = a * (e * before) - a * a / root * (e * open_a * x)
    df = dlog * log * (1 - open_f)
    drate = -(dlog * open_f).sum((0, 1))
    dstate = None
    if s["state"] is not None:
        if dense:
            dstate = a[0] * e[0]
        else:
            dstate = torch.where((count > 0)[:, None], (a * e)[first.clamp(max=a.shape[0] - 1), 0],
                                 s["dlast"] if s["dlast"] is not None else 0)
    return y, last, back(dx), back(df), back(da), drate, dstate


def _positions(s):
    if s["positions"] is not None:
        return s["positions"]
    at, seq, first, _ = _layout(s)
    return (at - first[seq]).reshape(s["q"].shape[:-2])


def _turn(v, cos, sin, interleaved):
    """Pairs of the first 2n values of each head turned by their angle."""
    n = cos.shape[-1]
    if interleaved:
        a, b = v[..., 0:2 * n:2], v[..., 1:2 * n:2]
    else:
        a, b = v[..., :n], v[..., n:2 * n]
    a, b = a * cos - b * sin, a * sin + b * cos
    pairs = torch.stack([a, b], -1).flatten(-2) if interleaved else torch.cat([a, b], -1)
    return torch.cat([pairs, v[..., 2 * n:]], -1)


def _plain_rotate(s):
    c, t = s["case"], s["q"].dtype
    angle = _positions(s).double()[..., None, None] * s["rates"].double()
    cos, sin = torch.cos(angle).float(), torch.sin(angle).float()
    outs, grads, weights = [], [], []
    for x, w, g in ((s["q"], s["q_weight"], s.get("dq")), (s["k"], s["k_weight"], s.get("dk"))):
        x = x.float()
        r = torch.rsqrt((x * x).mean(-1, keepdim=True) + EPS)
        n = x * r
        outs.append(_turn(n * w, cos, sin, c["interleaved"]).to(t))
        if g is not None:
            g = _turn(g.float(), cos, -sin, c["interleaved"])
            weights.append((g * n).reshape(-1, c["dim"]).sum(0))
            g = g * w
            grads.append((r * (g - n * (g * n).mean(-1, keepdim=True))).to(t))
    return (*outs, *grads, *weights)


def _ring(s, position):
    """The row of a cache entry that holds a position."""
    w, k = s["case"]["window"], s["case"]["sinks"]
    return torch.where(position < k, position, k + (position - k) % w)


def _plain_attend_token(s):
    c, t = s["case"], s["q"].dtype
    d, h, kv = c["dim"], c["heads"], c["kv_heads"]
    at, p = s["slots"].long(), s["positions"].long()
    s["cache"][0, at, _ring(s, p)] = s["k"]
    s["cache"][1, at, _ring(s, p)] = s["v"]
    k, v = (x[at].float().transpose(1, 2) for x in s["cache"].unbind(0))  # (batch, kv, seen, d)
    q = s["q"].float().reshape(-1, kv, h // kv, d) * d ** -0.5
    score = q @ k.transpose(-1, -2)
    held = torch.arange(k.shape[2], device="cuda") <= p[:, None, None, None]
    score = torch.where(held, score, -math.inf)
    e = torch.exp(score - score.max(-1, keepdim=True).values)
    return ((e / e.sum(-1, keepdim=True)) @ v).reshape(s["q"].shape).to(t), s["cache"]


def _plain_attend(s):
    """Blocks of n rows against their own keys and the block's before, n rows
    being a window; first tokens out of the window by themselves."""
    c, t = s["case"], s["q"].dtype
    d, h, kv = c["dim"], c["heads"], c["kv_heads"]
    g, rows = h // kv, _rows(c)
    n = min(c["window"], rows)
    blocks = -(-rows // n)
    at, seq, first, count = _layout(s)
    scale = d ** -0.5

    def own_rows(x, heads):  # (blocks, kv, heads / kv * n, d)
        x = torch.cat([x, x.new_zeros(blocks * n - rows, heads, d)])
        return x.reshape(blocks, n, kv, heads // kv, d).permute(0, 2, 3, 1, 4).reshape(blocks, kv, -1, d)

    def band(x):  # (blocks, kv, 2n, d): the block's before and its own
        x = own_rows(x, kv)
        return torch.cat([torch.cat([torch.zeros_like(x[:1]), x[:-1]]), x], 2)

    def whole_rows(x, heads):
        x = x.reshape(blocks, kv, heads // kv, n, d).permute(0, 3, 1, 2, 4)
        return x.reshape(blocks * n, heads, d)[:rows]

    q, k, v = (s[x].reshape(rows, -1, d).float() for x in ("q", "k", "v"))
    qb, kb, vb = own_rows(q * scale, h), band(k), band(v)
    i = torch.arange(blocks * n, device="cuda").reshape(blocks, n, 1)
    j = (torch.arange(blocks, device="cuda")[:, None] - 1) * n + torch.arange(2 * n, device="cuda")
    j = j[:, None]
    begin = torch.cat([first[seq], at.new_zeros(blocks * n - rows)]).reshape(blocks, n, 1)
    seen = (j <= i) & (i - j < c["window"]) & (j >= begin)
    seen = seen[:, None, None].expand(blocks, kv, g, n, 2 * n).reshape(blocks, kv, g * n, 2 * n)
    score = torch.where(seen, qb @ kb.transpose(-1, -2), -math.inf)
    top = score.max(-1, keepdim=True).values
    if c["sinks"]:
        lead = torch.arange(c["sinks"], device="cuda")
        sink = (first[seq][:, None] + lead).clamp(max=rows - 1)  # (rows, sinks)
        far = at[:, None] - sink >= c["window"]
        far = far & (lead < count[seq][:, None])

        def of_rows(x):  # (rows, kv, g, ..) to blocks
            x = torch.cat([x.reshape(rows, h, -1), x.new_zeros(blocks * n - rows, h, x.shape[-1])])
            return x.reshape(blocks, n, kv, g, -1).permute(0, 2, 3, 1, 4).reshape(blocks, kv, g * n, -1)

        ks, vs = k[sink].permute(0, 2, 1, 3), v[sink].permute(0, 2, 1, 3)  # (rows, kv, sinks, d)
        qs = q.reshape(rows, kv, g, d) * scale
        extra = torch.where(far[:, None, None], qs @ ks.transpose(-1, -2), -math.inf)
        extra = of_rows(extra)
        top = torch.maximum(top, extra.max(-1, keepdim=True).values)
    top = torch.where(top > -math.inf, top, 0)  # rows behind the last
    e = torch.exp(score.sub_(top))
    total = e.sum(-1, keepdim=True)
    if c["sinks"]:
        extra = torch.exp(extra - top)
        total = total + extra.sum(-1, keepdim=True)
        extra = extra / total
        xs = whole_rows_of(extra, blocks, kv, g, n, rows)
    p = e.div_(total)
    y = whole_rows(p @ vb, h)
    if c["sinks"]:
        y = y + (xs @ vs).reshape(rows, h, d)
    if c["op"] == "attend_prompt":
        # the rows that a next token still sees, at their places of the cache
        place = at - first[seq]
        kept = (place < c["sinks"]) | (count[seq] - place <= c["window"])
        entry, row = s["slots"].long()[seq[kept]], _ring(s, place[kept])
        s["cache"][0, entry, row] = s["k"].reshape(rows, kv, d)[kept]
        s["cache"][1, entry, row] = s["v"].reshape(rows, kv, d)[kept]
        return y.to(t).reshape(s["q"].shape), s["cache"]
    dy = s["dy"].reshape(rows, h, d).float()
    dyb = own_rows(dy, h)
    delta = own_rows((dy * y).contiguous(), h).sum(-1, keepdim=True)
    dv = p.transpose(-1, -2) @ dyb
    ds = p * (dyb @ vb.transpose(-1, -2) - delta)
    dq = whole_rows(ds @ kb, h) * scale
    dk = ds.transpose(-1, -2) @ qb

    def from_band(x):  # each block's keys: its own rows and the next block's look back
        x = x.reshape(blocks, kv, 2, n, d)
        x = x[:, :, 1] + torch.cat([x[1:, :, 0], torch.zeros_like(x[:1, :, 0])])
        return whole_rows(x, kv)

    dk, dv = from_band(dk), from_band(dv)
    if c["sinks"]:
        dyr = dy.reshape(rows, kv, g, d)
        dxs = xs * (dyr @ vs.transpose(-1, -2) - (dy * y).sum(-1).reshape(rows, kv, g, 1))
        dq = dq + (dxs @ ks).reshape(rows, h, d) * scale
        dk = dk.index_add(0, sink.reshape(-1), (dxs.transpose(-1, -2) @ qs).transpose(1, 2).reshape(-1, kv, d))
        dv = dv.index_add(0, sink.reshape(-1), (xs.transpose(-1, -2) @ dyr).transpose(1, 2).reshape(-1, kv, d))
    return tuple(x.to(t).reshape(s[like].shape)
                 for x, like in ((y, "q"), (dq, "q"), (dk, "k"), (dv, "v")))


def whole_rows_of(x, blocks, kv, g, n, rows):
    """(blocks, kv, g n, m) to (rows, kv, g, m)."""
    x = x.reshape(blocks, kv, g, n, -1).permute(0, 3, 1, 2, 4)
    return x.reshape(blocks * n, kv, g, -1)[:rows]


def run(state):
    if own:
        return _run_own(state)
    op = state["case"]["op"]
    if op.startswith("gated"):
        return _plain_gated(state)
    if op.startswith("rotate"):
        return _plain_rotate(state)
    return _plain_attend_token(state) if op == "attend_token" else _plain_attend(state)


# ------------------------------------------------- the definition in 64 bits
def _spans(s):
    c = s["case"]
    if s["offsets"] is None:
        n = c.get("length", 1)
        return [(i * n, (i + 1) * n) for i in range(c["batch"])]
    o = s["offsets"].tolist()
    return list(zip(o[:-1], o[1:]))


def _logistic(v):
    return 1 / (1 + torch.exp(-v))


def _exact_gated(s):
    """Row after row, all dense sequences at once or the packed rows in one run
    whose state changes hands where a sequence opens."""
    c = s["case"]
    ch, train = c["channels"], c["op"] == "gated_train"
    rate = s["rate"].double()
    if c["op"] == "gated_token":
        at = s["slots"].long()
        keep = torch.exp(-rate * _logistic(s["forget"].double()))
        state = s["state"].double()
        h = keep * state[at] + torch.sqrt(1 - keep ** 2) * _logistic(s["admit"].double()) * s["x"].double()
        state[at] = h
        return h, state
    dense = s["offsets"] is None
    order = (lambda v: v.double().transpose(0, 1)) if dense else (lambda v: v.double()[:, None])
    back = (lambda v: v.transpose(0, 1)) if dense else (lambda v: v[:, 0])
    x, f, i = order(s["x"]), _logistic(order(s["forget"])), _logistic(order(s["admit"]))
    keep = torch.exp(-rate * f)
    room = torch.sqrt(1 - keep ** 2)
    rows, width = x.shape[0], x.shape[1]
    zero = x.new_zeros(width, ch)
    h0 = s["state"].double() if s["state"] is not None else None
    spans = [(0, 0, rows)] if dense else [(n, lo, hi) for n, (lo, hi) in enumerate(_spans(s)) if hi > lo]
    opens, closes = {lo: n for n, lo, _ in spans}, {hi - 1: n for n, _, hi in spans}

    def of(v, n):
        return zero if v is None else v if dense else v[n:n + 1]

    hs, before = room * i * x, torch.empty_like(x)
    h = zero
    for t in range(rows):
        if t in opens:
            h = of(h0, opens[t])
        before[t] = h
        h = torch.addcmul(hs[t], keep[t], h, out=hs[t])
    if dense:
        last = hs[-1]
    else:
        last = h0.clone() if h0 is not None else x.new_zeros(c["batch"], ch)
        for n, _, hi in spans:
            last[n] = hs[hi - 1, 0]
    if not train:
        return back(hs), last
    dlast = s["dlast"].double() if s["dlast"] is not None else None
    e = order(s["dy"]).clone()
    dstate = None
    if h0 is not None:
        dstate = dlast.clone() if dlast is not None else x.new_zeros(c["batch"], ch)
    carry = zero
    for t in reversed(range(rows)):
        if t in closes:
            carry = of(dlast, closes[t])
        e[t] += carry
        carry = keep[t] * e[t]
        if t in opens and dstate is not None:
            dstate[slice(None) if dense else slice(opens[t], opens[t] + 1)] = carry
    dkeep = e * before - e * i * x * keep / room
    df = dkeep * keep * -rate
    return (back(hs), last, back(e * room * i), back(df * f * (1 - f)),
            back(e * room * x * i * (1 - i)), -(dkeep * keep * f).sum((0, 1)), dstate)


def _exact_rotate(s):
    """By complex numbers, the gradient by autograd."""
    c = s["case"]
    n, train = c["turned"] // 2, c["op"] == "rotate_train"
    if s["positions"] is not None:
        place = s["positions"].double()
    else:
        place = torch.cat([torch.arange(hi - lo, device="cuda") for lo, hi in _spans(s)])
        place = place.double().reshape(s["q"].shape[:-2])
    turn = torch.polar(torch.ones((), device="cuda", dtype=torch.float64),
                       place[..., None] * s["rates"].double()).unsqueeze(-2)
    outs, grads, weights = [], [], []
    for name in ("q", "k"):
        x = s[name].double().requires_grad_(train)
        w = s[name + "_weight"].double().requires_grad_(train)
        v = x / torch.sqrt((x ** 2).sum(-1, keepdim=True) / c["dim"] + EPS) * w
        head = v[..., :2 * n]
        pairs = head.unflatten(-1, (n, 2)) if c["interleaved"] else head.unflatten(-1, (2, n)).transpose(-1, -2)
        pairs = torch.view_as_real(torch.view_as_complex(pairs.contiguous()) * turn)
        head = pairs.flatten(-2) if c["interleaved"] else pairs.transpose(-1, -2).flatten(-2)
        y = torch.cat([head, v[..., 2 * n:]], -1)
        outs.append(y.detach())
        if train:
            gx, gw = torch.autograd.grad(y, (x, w), s["d" + name].double())
            grads.append(gx)
            weights.append(gw)
    return (*outs, *grads, *weights)


def _exact_attend_token(s):
    c = s["case"]
    d, w, sinks = c["dim"], c["window"], c["sinks"]
    cache = s["cache"].double()
    y = torch.empty(s["q"].shape, dtype=torch.float64, device="cuda")
    for b, (slot, p) in enumerate(zip(s["slots"].tolist(), s["positions"].tolist())):
        row = p if p < sinks else sinks + (p - sinks) % w
        cache[0, slot, row], cache[1, slot, row] = s["k"][b].double(), s["v"][b].double()
        k, v = cache[:, slot, :p + 1].repeat_interleave(c["heads"] // c["kv_heads"], dim=2)
        p = torch.softmax(torch.einsum("hd,nhd->hn", s["q"][b].double(), k) / math.sqrt(d), -1)
        y[b] = torch.einsum("hn,nhd->hd", p, v)
    return y, cache


def _exact_attend(s):
    """Sequence by sequence, some rows at a time against all that any of them sees."""
    c = s["case"]
    d, h, kv, w, sinks = (c[x] for x in ("dim", "heads", "kv_heads", "window", "sinks"))
    train, rows = c["op"] == "attend_train", _rows(c)
    q, k, v = (s[x].reshape(rows, -1, d).double() for x in ("q", "k", "v"))
    y = torch.zeros_like(q)
    grads = [torch.zeros_like(x) for x in (q, k, v)] if train else None
    for lo, hi in _spans(s):
        step = max(16, min(1024, int(1.5e8 / max(1, h * min(hi - lo, w + 1024)))))
        for a in range(lo, hi, step):
            b = min(hi, a + step)
            begin = max(lo, a - w + 1)
            js = torch.cat([torch.arange(lo, min(lo + sinks, begin), device="cuda"),
                            torch.arange(begin, b, device="cuda")])
            i = torch.arange(a, b, device="cuda")[:, None]
            hidden = (js > i) | ((i - js >= w) & (js - lo >= sinks))
            part = [x.requires_grad_(train) for x in (q[a:b].clone(), k[js], v[js])]
            qh = part[0].unflatten(1, (kv, h // kv))
            score = torch.einsum("ikgd,jkd->kgij", qh, part[1]) / math.sqrt(d)
            p = torch.softmax(score.masked_fill(hidden, -math.inf), -1)
            out = torch.einsum("kgij,jkd->ikgd", p, part[2]).flatten(1, 2)
            y[a:b] = out.detach()
            if train:
                got = torch.autograd.grad(out, part, s["dy"].reshape(rows, h, d)[a:b].double())
                grads[0][a:b] = got[0]
                grads[1][js] += got[1]
                grads[2][js] += got[2]
    if train:
        return tuple(x.reshape(s[like].shape) for x, like in zip((y, *grads), ("q", "q", "k", "v")))
    cache = s["cache"].double()
    for slot, (lo, hi) in zip(s["slots"].tolist(), _spans(s)):
        for p in list(range(min(sinks, hi - lo))) + list(range(max(sinks, hi - lo - w), hi - lo)):
            row = p if p < sinks else sinks + (p - sinks) % w
            cache[0, slot, row], cache[1, slot, row] = k[lo + p], v[lo + p]
    return y.reshape(s["q"].shape), cache


def exact(case, seed):
    s = prepare(case, seed)
    op = case["op"]
    if op.startswith("gated"):
        return _exact_gated(s)
    if op.startswith("rotate"):
        return _exact_rotate(s)
    return _exact_attend_token(s) if op == "attend_token" else _exact_attend(s)
