"""The gated recurrence at the ends of its range: states that are not finite,
decays next to one and far from it."""
import pytest
import torch

import mixing_reference as ref
from mixing_reference import TYPES, close, cuda, offsets_of, randn

gpu = pytest.mark.gpu


@pytest.fixture(scope="module")
def tcu():
    from paper_1908_06649_gb300 import _build
    _build.build()
    import paper_1908_06649_gb300 as p
    p.lib()
    return p


@gpu
@pytest.mark.parametrize("bad", [float("inf"), -float("inf"), float("nan")])
@pytest.mark.parametrize("channels", [6, 64 * 20])  # blocks of a cluster, blocks alone
def test_what_is_not_finite_stays_in_its_sequence(tcu, bad, channels):
    """Decays whose product over a warp's rows, or a tile's, is below fp32's
    range end no sequence: a state, an input or a gradient that is not finite
    reaches every later (earlier) row of its own sequence, packed as dense, and
    no other."""
    gen = torch.Generator().manual_seed(0)
    lengths = [50, 700, 60]
    off = offsets_of(lengths).cuda()
    x, dy = randn(gen, 2, sum(lengths), channels).cuda().unbind(0)
    open_ = torch.full_like(x, 8.0)
    rate = torch.linspace(0.05, 30, channels).cuda()
    state, dlast = randn(gen, 2, 3, channels).cuda().unbind(0)
    args = (open_, open_, rate)
    clean, end, marks = tcu.gated_scan(x, *args, state=state, offsets=off, marks=True)
    g = tcu.gated_scan_grad(dy, x, *args, marks=marks, state=state, offsets=off, dlast=dlast)
    for where in ("state", "x"):
        x2, state2 = x.clone(), state.clone()
        if where == "state":
            state2[1] = bad
        else:
            x2[53] = bad
        y, last, _ = tcu.gated_scan(x2, *args, state=state2, offsets=off, marks=True)
        assert torch.equal(y[:50], clean[:50]) and torch.equal(y[750:], clean[750:]), where
        assert not y[53:750].isfinite().any(), where
        assert torch.equal(last[::2], end[::2]) and not last[1].isfinite().any()
        alone, _ = tcu.gated_scan(x2[None, 50:750], open_[None, 50:750], open_[None, 50:750], rate,
                                  state=state2[1:2])
        assert not alone[:, 3:].isfinite().any()
    for where in ("dlast", "dy"):
        dy2, dlast2 = dy.clone(), dlast.clone()
        if where == "dlast":
            dlast2[1] = bad
        else:
            dy2[747] = bad
        b = tcu.gated_scan_grad(dy2, x, *args, marks=marks, state=state, offsets=off, dlast=dlast2)
        assert torch.equal(b.x[:50], g.x[:50]) and torch.equal(b.x[750:], g.x[750:]), where
        assert not b.x[50:748].isfinite().any(), where
        assert torch.equal(b.state[::2], g.state[::2]) and not b.state[1].isfinite().any()


@gpu
@pytest.mark.parametrize("kind", ["clusters", "blocks", "packed"])
def test_gates_that_hardly_change(tcu, kind):
    """Constant gates and decays within 5e-6 to 5e-4 of one over 30000 rows: a
    decay that is off in its last place, 2^-25 of one, is so at every row, and
    a state remembers 1 / (1 - a) of them.  Held as a - 1 it is 2^-22 of that
    off, as the special function unit's results are, and the state as much: with
    an input of the same sign and a factor of four for what multiplies it,
    1e-6; 2e-5 holds it, and the gradients."""
    rows, ch, batch = 30000, 64, 300 if kind == "blocks" else 1
    lengths = [rows] if kind != "packed" else [300, rows - 5000, 0, 4000, 700]
    gen = torch.Generator(device="cuda").manual_seed(0)
    r = lambda *s: torch.randn(*s, generator=gen, device="cuda")  # noqa: E731
    x, dy = r(batch, rows, ch) + 1, r(batch, rows, ch) + 1
    forget, admit = (torch.zeros(1, 1, ch, device="cuda") + g for g in (0.0, 1.0))
    forget, admit = forget.repeat(batch, rows, 1), admit.repeat(batch, rows, 1)
    rate = torch.logspace(-5, -3, ch, device="cuda")
    seqs = batch if kind != "packed" else len(lengths)
    state, dlast = r(seqs, ch), r(seqs, ch)
    more = {}
    if kind == "packed":
        x, dy, forget, admit = x[0], dy[0], forget[0], admit[0]
        more["offsets"] = offsets_of(lengths).cuda()
    y, last, marks = tcu.gated_scan(x, forget, admit, rate, state=state, marks=True, **more)
    g = tcu.gated_scan_grad(dy, x, forget, admit, rate, marks=marks, state=state, dlast=dlast, **more)
    off = [0]
    for n in lengths:
        off.append(off[-1] + n)
    for s in (0, batch - 1) if kind == "blocks" else range(seqs):  # of the blocks' entries two
        at = slice(off[s], off[s + 1]) if kind == "packed" else s
        if kind == "packed" and not lengths[s]:
            assert torch.equal(last[s], state[s]) and torch.equal(g.state[s], dlast[s])
            continue
        n = lengths[s] if kind == "packed" else rows
        xs, dys = x[at].double(), dy[at].double()
        log = -rate.double() / 2
        keep, room, way = torch.exp(log), torch.sqrt(-torch.expm1(2 * log)), torch.sigmoid(admit[at][0].double())
        new = room * way * xs
        h, before, hs = state[s].double(), torch.empty_like(xs), torch.empty_like(xs)
        for t in range(n):
            before[t] = h
            h = keep * h + new[t]
            hs[t] = h
        e, carry = torch.empty_like(xs), dlast[s].double()
        for t in reversed(range(n)):
            e[t] = dys[t] + carry
            carry = keep * e[t]
        dlog = keep * e * before - keep ** 2 / room * e * way * xs
        for j in range(0, ch, 9):  # each on its own: their sizes differ
            for got, want, name in (
                    (y[at], hs, "y"), (g.x[at], e * room * way, "dx"), (g.forget[at], dlog * log / 2, "dforget"),
                    (g.admit[at], e * room * xs * way * (1 - way), "dadmit")):
                close(got[..., j], want[..., j].cpu(), (name, s, j))
        close(last[s], h.cpu(), "last")
        close(g.state[s], carry.cpu(), "dstate")
    if batch == 1 and kind != "packed":
        close(g.rate, (dlog * log / rate).sum(0).cpu(), "drate")


@gpu
def test_tokens_of_gates_that_hardly_change(tcu):
    """The same, a token at a time."""
    ch, steps = 64, 3000
    gen = torch.Generator(device="cuda").manual_seed(0)
    x = torch.randn(steps, 1, ch, generator=gen, device="cuda") + 1
    gate = torch.zeros(1, ch, device="cuda")
    rate = torch.logspace(-4, 0, ch, device="cuda")
    state = torch.randn(1, ch, generator=gen, device="cuda") * 100
    log = -rate.double() / 2
    keep, room = torch.exp(log), torch.sqrt(-torch.expm1(2 * log))
    want = state.double()
    for t in range(steps):
        tcu.gated_scan_step(x[t], gate, gate, rate, state)
        want = keep * want + room / 2 * x[t].double()
    for j in range(ch):
        close(state[0, j:j + 1], want[0, j:j + 1].cpu(), j)


@gpu
def test_decays_far_from_one(tcu):
    """Rates that leave nothing of a state beside rates that leave nearly all of
    it: what a row forgets does not stay as a rounding of what it was."""
    ch = 64
    gen = torch.Generator().manual_seed(0)
    x = randn(gen, 1, 400, ch) * 10.0 ** -torch.arange(400)[:, None].div(20, rounding_mode="floor")
    forget, admit = randn(gen, 1, 400, ch) + 2, randn(gen, 1, 400, ch)
    rate = torch.logspace(0.5, 1.5, ch)
    rate[1::2] = torch.logspace(-3, -1, ch // 2)
    a = dict(x=x, forget=forget, admit=admit, rate=rate, state=randn(gen, 1, ch) * 1e4)
    y, _ = ref.gated(**{k: v.double() for k, v in a.items()})
    got, _ = tcu.gated_scan(**cuda(a))
    for t in range(0, 400, 20):  # inputs of one size at a time
        for part in (slice(0, None, 2), slice(1, None, 2)):
            close(got[0, t + 10:t + 20, part], y[0, t + 10:t + 20, part], (t, part))


@gpu
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("packed", [False, True])
@pytest.mark.parametrize("share", [16, 12, 9, 8, 6, 4, 3, 2])
def test_all_sizes_of_clusters(tcu, dtype, packed, share):
    """Channels for which a strip's rows are shared by 16, 12, 9, 8, 6, 4, 3 or 2
    blocks, over rows that take several exchanges between them, in sequences
    that open in different ones; some strips against the definition."""
    sms = torch.cuda.get_device_properties(0).multi_processor_count
    strips = (sms * 29 // 20 if share > 4 else sms * 9 // 5) // share
    ch, lengths = strips * 64, [5200] if not packed else [700, 0, 1, 2900, 133, 1466]
    rows, seqs = sum(lengths), len(lengths)
    gen = torch.Generator(device="cuda").manual_seed(share)
    r = lambda *s: torch.randn(*s, generator=gen, device="cuda")  # noqa: E731
    x, f, i, dy = (r(rows, ch).to(dtype) for _ in range(4))
    rate, state, dlast = torch.exp(r(ch) - 3), r(seqs, ch), r(seqs, ch)
    args = (x, f, i) if packed else (x[None], f[None], i[None])
    more = dict(offsets=offsets_of(lengths).cuda()) if packed else {}
    y, last, marks = tcu.gated_scan(*args, rate, state=state, marks=True, **more)
    g = tcu.gated_scan_grad(dy if packed else dy[None], *args, rate, marks=marks, state=state,
                            dlast=dlast, **more)
    some = torch.cat([torch.arange(64) + 64 * s for s in sorted({0, strips // 2, strips - 1})]).cuda()
    x, f, i, dy, dlast = (t[:, some].double() for t in (x, f, i, dy, dlast))
    log = -rate[some].double() * torch.sigmoid(f)
    keep, room, way = torch.exp(log), torch.sqrt(-torch.expm1(2 * log)), torch.sigmoid(i)
    before, hs, e = (torch.empty_like(keep) for _ in range(3))
    ends, starts, at = [], [], 0
    for s, n in enumerate(lengths):
        h = state[s, some].double()
        for t in range(at, at + n):
            before[t] = h
            h = keep[t] * h + room[t] * way[t] * x[t]
            hs[t] = h
        ends.append(h)
        carry = dlast[s]
        for t in reversed(range(at, at + n)):
            e[t] = dy[t] + carry
            carry = keep[t] * e[t]
        starts.append(carry)
        at += n
    dlog = keep * e * before - keep ** 2 / room * e * way * x
    rows_of = lambda t: (t if packed else t[0])[:, some]  # noqa: E731
    close(rows_of(y), hs.cpu(), "y")
    close(last[:, some], torch.stack(ends).cpu(), "last")
    close(rows_of(g.x), (e * room * way).cpu(), "dx")
    close(rows_of(g.admit), (e * room * x * way * (1 - way)).cpu(), "dadmit")
    close(rows_of(g.forget), (dlog * log * (1 - torch.sigmoid(f))).cpu(), "dforget")
    close(g.rate[some], (dlog * log / rate[some]).sum(0).cpu(), "drate")
    close(g.state[:, some], torch.stack(starts).cpu(), "dstate")
