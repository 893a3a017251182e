"""The gated linear recurrence on the GPU against its definition in 64 bits
(mixing_reference.py), through the package's calls; and what it refuses.

Tolerances, set before the first run.  The arithmetic before the one rounding
of an output is fp32: 2^x and reciprocals by the special function unit are
2^-22 off, so a decay is 2^-22 off at most and a product of m of them sqrt(m)
times that for errors of random sign; with m <= 1100 rows here, 8e-6; the
default of 2e-5 leaves a factor of two for the sums."""
import ctypes

import pytest
import torch

import mixing_reference as ref
from mixing_reference import TYPES, close, cuda, doubled, offsets_of, packed_lengths, randn

gpu = pytest.mark.gpu
NAMES = ("x", "forget", "admit", "rate", "state")


@pytest.fixture(scope="module")
def tcu():
    from paper_1908_06649_gb300 import _build
    _build.build()
    import paper_1908_06649_gb300 as p
    p.lib()
    return p


def inputs(dtype, lead, ch, seqs, state=True, seed=0, offsets=None):
    gen = torch.Generator().manual_seed(seed)
    r = lambda *s, **k: randn(gen, *s, **k)  # noqa: E731
    a = dict(x=r(*lead, ch, dtype=dtype), forget=r(*lead, ch, dtype=dtype, scale=2),
             admit=r(*lead, ch, dtype=dtype), rate=torch.exp(r(ch) - 2),
             state=r(seqs, ch) if state else None, offsets=offsets)
    return a, r(*lead, ch, dtype=dtype), r(seqs, ch)


def check(tcu, a, dy, dlast):
    d = doubled(a, NAMES)
    y, last = ref.gated(**d)
    leaves = [d[n] for n in NAMES if d[n] is not None]
    grads = list(torch.autograd.grad((y, last), leaves, (dy.double(), dlast.double()),
                                     allow_unused=True))
    c = cuda(a)
    got, end, marks = tcu.gated_scan(**c, marks=True)
    close(got, y, "y")
    close(end, last, "last")
    assert torch.equal(tcu.gated_scan(**c)[0], got)
    g = tcu.gated_scan_grad(dy.cuda(), **c, marks=marks, dlast=dlast.cuda())
    again = tcu.gated_scan_grad(dy.cuda(), **c, marks=marks, dlast=dlast.cuda())
    for n in NAMES:
        if a[n] is None:
            assert getattr(g, n) is None
            continue
        close(getattr(g, n), grads.pop(0), "d" + n)
        assert torch.equal(getattr(g, n), getattr(again, n)), n


@gpu
@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("batch,length,ch,state", [
    (1, 1, 1, False), (2, 1, 64, True), (3, 37, 65, True), (2, 130, 96, False), (1, 8, 2, True),
    (2, 64, 130, True), (1, 1100, 34, True), (5, 9, 7, False)])
def test_dense(tcu, dtype, batch, length, ch, state):
    check(tcu, *inputs(dtype, (batch, length), ch, batch, state))


@gpu
@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("kind", ["one", "empties", "singles", "mixed"])
@pytest.mark.parametrize("total,ch,state", [(77, 66, True), (1090, 33, False)])
def test_packed(tcu, dtype, kind, total, ch, state):
    lengths = packed_lengths(total, kind)
    check(tcu, *inputs(dtype, (total,), ch, len(lengths), state, offsets=offsets_of(lengths)))


@gpu
def test_many_short_sequences(tcu):
    lengths = [k % 3 for k in range(900)]
    check(tcu, *inputs(torch.float32, (sum(lengths),), 6, 900, True, offsets=offsets_of(lengths)))


@gpu
@pytest.mark.parametrize("dtype", TYPES)
def test_strides(tcu, dtype):
    """Slices of one projection, of odd starts, batch entries apart or in
    another order: the same bits as their copies."""
    gen = torch.Generator().manual_seed(3)
    for wide, at, ch in ((256, (0, 64, 128), 64), (199, (1, 66, 133), 65), (200, (2, 66, 130), 62)):
        big = randn(gen, 70, 3, wide, dtype=dtype).cuda().transpose(0, 1)
        rows = [big[..., i:i + ch] for i in at]
        rate = torch.rand(ch, generator=gen).cuda()
        y, last, marks = tcu.gated_scan(*rows, rate, marks=True)
        flat = [r.contiguous() for r in rows]
        y2, last2 = tcu.gated_scan(*flat, rate)
        assert torch.equal(y, y2) and torch.equal(last, last2)
        g = tcu.gated_scan_grad(rows[0], *rows, rate, marks=marks)
        for got, want in zip(g, tcu.gated_scan_grad(flat[0], *flat, rate, marks=marks)):
            assert got is want is None or torch.equal(got, want)
        out = torch.zeros(3, 70, wide, dtype=dtype, device="cuda")
        tcu.gated_scan(*rows, rate, out=out[..., 1:1 + ch])
        assert torch.equal(out[..., 1:1 + ch], y) and out[..., 0].eq(0).all()


@gpu
@pytest.mark.parametrize("dtype", TYPES)
def test_ends_of_the_gates(tcu, dtype):
    """Gates shut and open to the last: the state stays, or only the input is left."""
    inf = float("inf")
    v = torch.tensor([-inf, -300.0, -90.0, -20.0, 0.0, 20.0, 90.0, 300.0, inf])
    ch = v.numel() ** 2
    forget, admit = (v.repeat_interleave(9), v.repeat(9))
    gen = torch.Generator().manual_seed(1)
    a = dict(x=randn(gen, 1, 5, ch, dtype=dtype), forget=forget.expand(1, 5, ch).to(dtype),
             admit=admit.expand(1, 5, ch).to(dtype), rate=torch.full((ch,), 3.0),
             state=randn(gen, 1, ch))
    d = doubled(a)
    y, last = ref.gated(**d)
    c = cuda(a)
    got, end, marks = tcu.gated_scan(**c, marks=True)
    close(got, y)
    close(end, last)
    g = tcu.gated_scan_grad(c["x"], **c, marks=marks)
    for n in NAMES:
        assert torch.isfinite(getattr(g, n)).all(), n
    shut = forget <= -90  # decays of one: e is the sum of dy
    want = a["x"].double().flip(1).cumsum(1).flip(1)[0, 0]
    close(g.state[0].cpu()[shut], want[shut])
    assert (g.forget[0].cpu()[:, torch.isinf(forget)] == 0).all()


@gpu
def test_decays_near_one(tcu):
    """1 - a^2 from decays within 1e-6 of one keeps its relative accuracy."""
    ch = 64
    gen = torch.Generator().manual_seed(2)
    a = dict(x=randn(gen, 2, 200, ch), forget=randn(gen, 2, 200, ch), admit=randn(gen, 2, 200, ch),
             rate=torch.logspace(-7, 1, ch), state=None)
    d = doubled(a, ("rate",))
    y, last = ref.gated(**d)
    c = cuda(a)
    got, end, marks = tcu.gated_scan(**c, marks=True)
    for j in range(ch):  # each channel on its own: their sizes differ
        close(got[..., j], y[..., j], j)
    (want,) = torch.autograd.grad(y, (d["rate"],), torch.ones_like(y))
    close(tcu.gated_scan_grad(torch.ones_like(c["x"]), **c, marks=marks).rate / want.float().cuda(),
          torch.ones_like(want))


@gpu
def test_sequences_do_not_reach_each_other(tcu):
    """What is not finite stays in its own sequence, forward and backward."""
    nan = float("nan")
    a, dy, dlast = inputs(torch.float32, (60,), 10, 3, True, offsets=offsets_of([20, 20, 20]))
    c, dy = cuda(a), dy.cuda()
    clean, _, marks = tcu.gated_scan(**c, marks=True)
    want = tcu.gated_scan_grad(dy, **c, marks=marks)
    for n in ("x", "forget", "admit"):
        c[n][20:40] = nan
    c["state"][1] = nan
    dy[20:40] = nan
    y, last, marks = tcu.gated_scan(**c, marks=True)
    g = tcu.gated_scan_grad(dy, **c, marks=marks)
    for rows in (slice(0, 20), slice(40, 60)):
        assert torch.equal(y[rows], clean[rows])
        for n in ("x", "forget", "admit"):
            assert torch.equal(getattr(g, n)[rows], getattr(want, n)[rows])
    assert torch.equal(g.state[::2], want.state[::2]) and torch.isfinite(last[::2]).all()


@gpu
@pytest.mark.parametrize("dtype", TYPES)
def test_rows_behind_the_last_sequence(tcu, dtype):
    """A padded pack: they are not written, and have no part in any gradient."""
    nan = float("nan")
    a, dy, dlast = inputs(dtype, (90,), 12, 2, True, offsets=offsets_of([30, 40]))
    short = {k: v[:70] if k in ("x", "forget", "admit") else v for k, v in a.items()}
    c, s = cuda(a), cuda(short)
    for n in ("x", "forget", "admit"):
        c[n][70:] = nan
    dy = dy.cuda()
    dy[70:] = nan
    out = torch.full_like(c["x"], 7.0)
    y, last, marks = tcu.gated_scan(**c, marks=True, out=out)
    y2, last2, marks2 = tcu.gated_scan(**s, marks=True)
    assert torch.equal(out[:70], y2) and (out[70:] == 7).all() and torch.equal(last, last2)
    g = tcu.gated_scan_grad(dy, **c, marks=marks, dlast=dlast.cuda())
    g2 = tcu.gated_scan_grad(dy[:70], **s, marks=marks2, dlast=dlast.cuda())
    for n in ("x", "forget", "admit"):
        assert torch.equal(getattr(g, n)[:70], getattr(g2, n)) and (getattr(g, n)[70:] == 0).all()
    assert torch.equal(g.rate, g2.rate) and torch.equal(g.state, g2.state)


@gpu
def test_no_rows_no_sequences_no_channels(tcu):
    for dtype in TYPES:
        x = torch.zeros(2, 0, 4, dtype=dtype, device="cuda")
        rate, state = torch.ones(4, device="cuda"), torch.rand(2, 4, device="cuda")
        y, last, marks = tcu.gated_scan(x, x, x, rate, state=state, marks=True)
        assert y.shape == x.shape and torch.equal(last, state)
        g = tcu.gated_scan_grad(x, x, x, x, rate, marks=marks, state=state, dlast=state)
        assert torch.equal(g.state, state) and (g.rate == 0).all()
        assert (tcu.gated_scan(x, x, x, rate)[1] == 0).all()
        none = torch.zeros(0, 4, dtype=dtype, device="cuda")
        off = torch.zeros(1, dtype=torch.int32, device="cuda")
        y, last = tcu.gated_scan(none, none, none, rate, offsets=off)
        assert y.shape == (0, 4) and last.shape == (0, 4)
        thin = torch.zeros(2, 3, 0, dtype=dtype, device="cuda")
        y, last = tcu.gated_scan(thin, thin, thin, rate[:0])
        assert y.shape == (2, 3, 0) and last.shape == (2, 0)


@gpu
@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("ch", [1, 64, 257])
def test_tokens_continue_a_prompt(tcu, dtype, ch):
    a, _, _ = inputs(dtype, (4, 21), ch, 4, False)
    c = cuda(a)
    y, last = tcu.gated_scan(**c)
    rows = lambda lo, hi: {n: c[n][:, lo:hi] for n in ("x", "forget", "admit")}  # noqa: E731
    _, state = tcu.gated_scan(**rows(0, 18), rate=c["rate"])
    cache = torch.full((9, ch), 5.0, device="cuda")
    slots = torch.tensor([7, 0, 3, 8], dtype=torch.int32, device="cuda")
    cache[slots.long()] = state
    for t in range(18, 21):
        one = {n: c[n][:, t] for n in ("x", "forget", "admit")}  # rows at the prompt's pitch
        step = tcu.gated_scan_step(**one, rate=c["rate"], state=cache, slots=slots)
        close(step, y[:, t].cpu().double(), inner=4 * ref.U[dtype] + 2e-5)
    close(cache[slots.long()], last.cpu().double())
    rest = [i for i in range(9) if i not in (7, 0, 3, 8)]
    assert (cache[rest] == 5).all()


@gpu
def test_tokens_of_slots_outside(tcu):
    gen = torch.Generator().manual_seed(0)
    x = randn(gen, 3, 6).cuda()
    cache = torch.ones(2, 6, device="cuda")
    slots = torch.tensor([-1, 1, 2], dtype=torch.int32, device="cuda")
    y = tcu.gated_scan_step(x, x, x, torch.ones(6, device="cuda"), cache, slots=slots)
    assert (y[0] == 0).all() and (y[2] == 0).all() and (y[1] != 0).all()
    assert (cache[0] == 1).all() and torch.equal(cache[1], y[1])
    # a token's row may replace one that it reads
    z = x.clone()
    tcu.gated_scan_step(z, x, x, torch.ones(6, device="cuda"), torch.ones(2, 6, device="cuda"),
                        slots=slots, out=z)
    assert torch.equal(z, y)


@gpu
@pytest.mark.parametrize("packed", [False, True])
def test_autograd_and_differences(tcu, packed):
    """Through autograd, and along a direction by central differences (h^2 of
    the third derivative and 2^-24 / h of the value: 1e-3 at h = 1e-2)."""
    off = offsets_of([3, 0, 30, 7]).cuda() if packed else None
    a, dy, dlast = inputs(torch.float32, (40,) if packed else (2, 20), 9, 4 if packed else 2,
                          offsets=off)
    c = cuda(a)
    leaves = {n: c[n].clone().requires_grad_() for n in NAMES}
    y, last = tcu.gated_scan(**leaves, offsets=off)
    ((y * dy.cuda()).sum() + (last * dlast.cuda()).sum()).backward()
    _, _, marks = tcu.gated_scan(**c, marks=True)
    g = tcu.gated_scan_grad(dy.cuda(), **c, marks=marks, dlast=dlast.cuda())
    gen = torch.Generator().manual_seed(9)
    for n in NAMES:
        assert torch.equal(leaves[n].grad, getattr(g, n)), n
        way = randn(gen, *c[n].shape).cuda() * (c[n] if n == "rate" else 1)

        def loss(h):
            y, last = tcu.gated_scan(**dict(c, **{n: c[n] + h * way}))
            return ((y * dy.cuda()).double().sum() + (last * dlast.cuda()).double().sum()).item()

        slope = (loss(1e-2) - loss(-1e-2)) / 2e-2
        want = (getattr(g, n).double() * way.double()).sum().item()
        scale = (getattr(g, n).double() * way.double()).norm().item()
        assert abs(slope - want) <= 2e-3 * max(abs(want), scale), n


@gpu
def test_graphs_and_streams(tcu):
    a, dy, dlast = inputs(torch.bfloat16, (300,), 130, 4, offsets=offsets_of([100, 0, 150, 50]))
    c, dy = cuda(a), dy.cuda()
    want = tcu.gated_scan(**c, marks=True)
    grads = tcu.gated_scan_grad(dy, **c, marks=want[2])
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    got = tcu.gated_scan(**c, marks=True, stream=side)
    torch.cuda.current_stream().wait_stream(side)
    for x, y in zip(got, want):
        assert torch.equal(x, y)
    token = {n: c[n][:4].clone() for n in ("x", "forget", "admit")}
    cache = c["state"].clone()
    with torch.cuda.stream(side):
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=side):
            y, last, marks = tcu.gated_scan(**c, marks=True)
            g = tcu.gated_scan_grad(dy, **c, marks=marks)
            step = tcu.gated_scan_step(**token, rate=c["rate"], state=cache)
    for _ in range(2):
        cache.copy_(c["state"])
        for t in (y, last, marks, *g):
            t.fill_(3)
        graph.replay()
        torch.cuda.synchronize()
        for x, w in zip((y, last, marks, *g), (*want, *grads)):
            assert torch.equal(x, w)
        fresh = c["state"].clone()
        assert torch.equal(step, tcu.gated_scan_step(**token, rate=c["rate"], state=fresh))
        assert torch.equal(cache, fresh)


@gpu
@pytest.mark.parametrize("batch,length,ch", [(1, 5000, 64), (2, 3000, 128), (300, 70, 64), (1, 40000, 2)])
def test_long_rows(tcu, batch, length, ch):
    """All sizes of clusters, against the recurrence in 64 bits on the GPU."""
    gen = torch.Generator(device="cuda").manual_seed(0)
    r = lambda *s: torch.randn(*s, generator=gen, device="cuda")  # noqa: E731
    x, f, i, dy = (r(batch, length, ch) for _ in range(4))
    rate, state, dlast = torch.exp(r(ch) - 2), r(batch, ch), r(batch, ch)
    y, last, marks = tcu.gated_scan(x, f, i, rate, state=state, marks=True)
    g = tcu.gated_scan_grad(dy, x, f, i, rate, marks=marks, state=state, dlast=dlast)
    log = -rate.double() * torch.sigmoid(f.double())
    keep, room = torch.exp(log), torch.sqrt(-torch.expm1(2 * log))
    way = torch.sigmoid(i.double())
    h, before, hs = state.double(), torch.empty_like(keep), torch.empty_like(keep)
    for t in range(length):
        before[:, t] = h
        h = keep[:, t] * h + room[:, t] * way[:, t] * x[:, t]
        hs[:, t] = h
    close(y, hs.cpu())
    close(last, h.cpu())
    e, carry = torch.empty_like(keep), dlast.double()
    for t in reversed(range(length)):
        e[:, t] = dy[:, t] + carry
        carry = keep[:, t] * e[:, t]
    dlog = keep * e * before - keep ** 2 / room * e * way * x
    close(g.state, carry.cpu())
    close(g.x, (e * room * way).cpu())
    close(g.admit, (e * room * x * way * (1 - way)).cpu())
    close(g.forget, (dlog * log * (1 - torch.sigmoid(f.double()))).cpu())
    close(g.rate, (dlog * log / rate).sum((0, 1)).cpu())


# ------------------------------------------------------------ without a GPU
@pytest.mark.parametrize("packed", [False, True])
def test_reference_against_differences(packed):
    gen = torch.Generator().manual_seed(0)
    off = offsets_of([2, 0, 3]) if packed else None
    lead, seqs = ((6,), 3) if packed else ((2, 3), 2)
    r = lambda *s: torch.randn(*s, generator=gen, dtype=torch.float64)  # noqa: E731
    args = [r(*lead, 2) for _ in range(3)] + [torch.exp(r(2)), r(seqs, 2)]
    assert torch.autograd.gradcheck(lambda *a: ref.gated(*a, offsets=off),
                                    [a.requires_grad_() for a in args])


def args(seq, **change):
    fake = 0x10000  # never dereferenced: every call here is refused
    r = seq._Rows(fake, 40, 8)
    v = dict(type=0, sequences=2, rows=5, channels=8, rate=fake, marks=fake, drate=fake, last=fake,
             workspace=fake, workspace_bytes=1 << 30,
             **{k: r for k in ("x", "forget", "admit", "y", "dy", "dx", "dforget", "dadmit")})
    v.update(change)
    return seq._GatedArgs(**v)


INVALID, UNSUPPORTED = 1, 2


@pytest.mark.parametrize("call,change,status", [
    ("", dict(type=3), INVALID), ("", dict(rows=-1), INVALID), ("", dict(channels=0), INVALID),
    ("", dict(sequences=-1), INVALID), ("", dict(rows=2 ** 31), UNSUPPORTED),
    ("", dict(channels=2 ** 31), UNSUPPORTED), ("", dict(rate=None), INVALID),
    ("", dict(rate=0x10002), INVALID), ("", dict(state=0x10001), INVALID),
    ("", dict(offsets=0x10000, workspace_bytes=4), INVALID),
    ("_grad", dict(marks=None), INVALID), ("_grad", dict(drate=None), INVALID),
    ("_grad", dict(workspace_bytes=8), INVALID), ("_grad", dict(dlast=0x10002), INVALID),
    ("_step", dict(), INVALID), ("_step", dict(rows=1, num_slots=1), INVALID),
    ("_step", dict(rows=1, num_slots=2, last=None), INVALID),
    ("_step", dict(rows=1, num_slots=2), INVALID),  # the cache over its rows
    ("_step", dict(rows=1, num_slots=2, offsets=0x10000), INVALID)])
def test_refusals(tcu, call, change, status):
    from paper_1908_06649_gb300 import sequence as seq
    assert getattr(seq._lib(), "tcu_gated_scan" + call)(args(seq, **change), None) == status


def test_refused_rows(tcu):
    from paper_1908_06649_gb300 import sequence as seq
    far, odd = seq._Rows(0x10000, 2 ** 33, 2 ** 31), seq._Rows(0x10001, 40, 8)
    for k in ("x", "forget", "admit", "y"):
        assert seq._lib().tcu_gated_scan(args(seq, **{k: far}), None) == UNSUPPORTED
        assert seq._lib().tcu_gated_scan(args(seq, **{k: odd}), None) == INVALID
    for k in ("dy", "dx", "dforget", "dadmit"):
        assert seq._lib().tcu_gated_scan_grad(args(seq, **{k: odd}), None) == INVALID
    assert seq._lib().tcu_gated_scan(None, None) == INVALID
    assert seq._lib().tcu_gated_scan_grad_workspace(args(seq)) > 0
    assert seq._lib().tcu_gated_scan_workspace(args(seq, channels=0)) == -1


def test_layout_of_the_arguments(tcu, tmp_path):
    import os
    import subprocess
    from paper_1908_06649_gb300 import _build, sequence as seq
    src, exe = tmp_path / "p.c", tmp_path / "p"
    src.write_text('#include <stddef.h>\n#include <stdio.h>\n#include "tcu_seq.h"\n'
                   "int main(void) { typedef tcu_gated_scan_args A; printf(\"%zu %zu %zu %zu\\n\","
                   "sizeof(A), offsetof(A, rate), offsetof(A, drate), offsetof(A, num_slots));"
                   "return 0; }\n")
    subprocess.run(["gcc", "-std=c99", "-Wall", "-Werror", "-I", os.path.dirname(_build.SEQ_HDR),
                    str(src), "-o", str(exe)], check=True)
    a = seq._GatedArgs
    got = subprocess.run([str(exe)], capture_output=True, text=True, check=True).stdout.split()
    assert list(map(int, got)) == [ctypes.sizeof(a), a.rate.offset, a.drate.offset, a.num_slots.offset]


def test_refusals_of_tensors(tcu):
    x, rate = torch.zeros(2, 5, 8), torch.zeros(8)
    with pytest.raises(ValueError):
        tcu.gated_scan(x, x, x, rate)
    with pytest.raises(TypeError):
        tcu.gated_scan(None, x, x, rate)
    with pytest.raises(ValueError):
        tcu.gated_scan_step(x[0], x[0], x[0], rate, torch.zeros(2, 8))


@gpu
def test_refusals_of_cuda_tensors(tcu):
    x, rate = torch.zeros(2, 5, 8, device="cuda"), torch.ones(8, device="cuda")
    y, last, marks = tcu.gated_scan(x, x, x, rate, marks=True)
    for bad in (dict(forget=x[:, :4]), dict(admit=x.half()), dict(rate=rate[:7]), dict(rate=rate.double()),
                dict(state=torch.zeros(3, 8, device="cuda")), dict(forget=x.cpu()),
                dict(x=x.transpose(1, 2)), dict(out=x), dict(out=x[:, :4]),
                dict(offsets=torch.zeros(3, dtype=torch.int32, device="cuda"))):
        with pytest.raises((ValueError, TypeError)):
            tcu.gated_scan(**{**dict(x=x, forget=x, admit=x, rate=rate), **bad})
    with pytest.raises(ValueError):
        tcu.gated_scan_grad(x, x, x, x, rate, marks=marks[:, :0])
    with pytest.raises(ValueError):
        tcu.gated_scan(x.requires_grad_(), x, x, rate, out=torch.zeros_like(x))
    x = x.detach()
    cache = torch.zeros(2, 8, device="cuda")
    for bad in (dict(state=cache[:1]), dict(state=cache.half()), dict(out=cache),
                dict(state=cache.clone().requires_grad_()), dict(x=cache),
                dict(slots=torch.zeros(2, dtype=torch.int64, device="cuda"))):
        a = dict(x=x[:, 0], forget=x[:, 0], admit=x[:, 0], rate=rate, state=cache)
        with pytest.raises((ValueError, TypeError, tcu.TcuDftError)):
            tcu.gated_scan_step(**{**a, **bad})
    from torch.autograd import forward_ad
    with forward_ad.dual_level():
        dual = forward_ad.make_dual(x, torch.ones_like(x))
        for call in (lambda: tcu.gated_scan(dual, x, x, rate),
                     lambda: tcu.gated_scan_grad(x, x, dual, x, rate, marks=marks),
                     lambda: tcu.gated_scan_step(x[:, 0], x[:, 0], dual[:, 0], rate, cache)):
            with pytest.raises(ValueError, match="forward-mode"):
                call()


@gpu
def test_beyond_32_bits_of_elements(tcu):
    """2.1e9 values a tensor: the end of a run is what a second call gives that
    continues from the first's last state."""
    rows, ch, cut = 525000, 4096, 524000
    gen = torch.Generator(device="cuda").manual_seed(0)
    x = torch.empty(1, rows, ch, dtype=torch.bfloat16, device="cuda").normal_(generator=gen)
    rate = torch.full((ch,), 0.5, device="cuda")
    y, last = tcu.gated_scan(x, x, x, rate)
    _, state = tcu.gated_scan(x[:, :cut], x[:, :cut], x[:, :cut], rate)
    end = x[:, cut:].clone()
    z, stop, marks = tcu.gated_scan(end, end, end, rate, state=state, marks=True)
    close(y[:, cut:], z.double().cpu(), inner=ref.U[torch.bfloat16] + 2e-5)
    close(last, stop.double().cpu())
    del y
    _, _, kept = tcu.gated_scan(x, x, x, rate, marks=True)
    g = tcu.gated_scan_grad(x, x, x, x, rate, marks=kept)
    w = tcu.gated_scan_grad(end, end, end, end, rate, marks=marks, state=state)
    close(g.forget[:, cut:], w.forget.double().cpu(), inner=ref.U[torch.bfloat16] + 2e-5)
