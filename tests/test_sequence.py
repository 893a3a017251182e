"""The sequence operators on the GPU against their definitions in 64 bits
(sequence_reference.py), through the package's calls.

Tolerances, set before the first run.  Outputs are rounded once to their
type: relative error at most u = 2^-8 (bf16), 2^-11 (f16), 2^-24 (f32).  The
arithmetic before it is fp32: 2^x by the special function unit is 2^-22 off,
an argument z adds z 2^-23, and a state is a product of up to m decays: with
errors of random sign their sum grows like 2^-22 sqrt(m / 3), 2.4e-6 at the
longest sequences here (m <= 300); 2e-5 leaves the sums over states, channels
and rows a factor of 8.  So the 2-norm of the error is within u + 2e-5 of the
result's; a value may lie on the other side of a rounding boundary, 2 u of
itself, plus 1e-4 of the result's root mean square."""
import pytest
import torch

import sequence_reference as ref

pytestmark = pytest.mark.gpu

U = {torch.float32: 2.0 ** -24, torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11}
TYPES = [torch.float32, torch.bfloat16, torch.float16]


@pytest.fixture(scope="module")
def pkg():
    from paper_1908_06649_gb300 import _build
    _build.build()
    import paper_1908_06649_gb300 as p
    p.lib()
    assert torch.cuda.is_available()
    return p


def close(got, want, name=""):
    assert got.shape == want.shape, name
    if not want.numel():
        return
    u = U[got.dtype]
    g, w = got.detach().cpu().double(), want.detach().double()
    err = (g - w).abs()
    norm = w.norm()
    assert torch.isfinite(g).all(), name
    assert err.norm() <= (u + 2e-5) * norm + 1e-30, (name, float(err.norm() / norm))
    rms = norm / w.numel() ** 0.5
    over = err - (2 * u * w.abs() + 1e-4 * rms)
    assert over.max() <= 1e-30, (name, float(over.max()), float(rms))


def randn(gen, *shape, dtype=torch.float32, scale=1.0):
    return (torch.randn(*shape, generator=gen) * scale).to(dtype)


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


# -------------------------------------------------------------- convolution
def conv_inputs(dtype, shape, width, packed, bias, state, seed=0):
    gen = torch.Generator().manual_seed(seed)
    ch = shape[-1]
    off = offsets_of(packed_lengths(shape[0], packed)) if packed else None
    seqs = len(off) - 1 if packed else shape[0]
    d = {"x": randn(gen, *shape, dtype=dtype),
         "weight": randn(gen, ch, width, scale=width ** -0.5),
         "bias": randn(gen, ch, scale=0.3) if bias else None,
         "state": randn(gen, seqs, width - 1, ch, dtype=dtype) if state else None,
         "offsets": off}
    d["dy"] = randn(gen, *shape, dtype=dtype)
    d["dlast"] = randn(gen, seqs, width - 1, ch, dtype=dtype)
    return d


def check_conv(pkg, d, act, dlast=True):
    c = cuda(d)
    args = (c["x"], c["weight"], c["bias"])
    more = {"silu": act, "state": c["state"], "offsets": c["offsets"]}
    y, last = pkg.short_conv(*args, **more)
    g = pkg.short_conv_grad(c["dy"], *args, dlast=c["dlast"] if dlast else None, **more)
    leaf = {k: d[k].double().requires_grad_() if d[k] is not None else None
            for k in ("x", "weight", "bias", "state")}
    ry, rl = ref.conv(leaf["x"], leaf["weight"], leaf["bias"], act, leaf["state"], d["offsets"])
    close(y, ry, "y")
    close(last, rl, "last")
    names = [k for k in leaf if leaf[k] is not None]
    loss = (ry * d["dy"].double()).sum()
    if dlast:
        loss = loss + (rl * d["dlast"].double()).sum()
    if not loss.requires_grad:
        loss = loss + sum(leaf[k].sum() * 0 for k in names)
    grads = torch.autograd.grad(loss, [leaf[k] for k in names], allow_unused=True)
    for k, w in zip(names, grads):
        close(getattr(g, k), w if w is not None else torch.zeros_like(leaf[k]), "d" + k)
    for k in ("bias", "state"):
        assert (getattr(g, k) is None) == (d[k] is None)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("width", [1, 2, 3, 4, 5, 7, 8])
@pytest.mark.parametrize("shape,packed", [
    ((2, 37, 48), None), ((1, 1, 16), None), ((3, 2, 33), None), ((2, 71, 7), None),
    ((1, 200, 64), None), ((97, 40), "mixed"), ((60, 17), "empties"), ((50, 24), "singles")])
def test_conv(pkg, dtype, width, shape, packed):
    check_conv(pkg, conv_inputs(dtype, shape, width, packed, width % 2 == 0, True), True)


@pytest.mark.parametrize("act", [False, True])
@pytest.mark.parametrize("bias", [False, True])
@pytest.mark.parametrize("state", [False, True])
@pytest.mark.parametrize("packed", [None, "mixed"])
def test_conv_options(pkg, act, bias, state, packed):
    shape = (133, 40) if packed else (2, 67, 40)
    d = conv_inputs(torch.bfloat16, shape, 4, packed, bias, state, seed=3)
    check_conv(pkg, d, act, dlast=state)


@pytest.mark.parametrize("packed", [None, "empties"])
def test_conv_of_no_rows(pkg, packed):
    d = conv_inputs(torch.float32, (0, 24) if packed else (2, 0, 24), 4, packed, True, True)
    check_conv(pkg, d, True)


@pytest.mark.parametrize("dtype", TYPES)
def test_conv_of_slices(pkg, dtype):
    """Rows inside a wider projection: strides and alignments of their own."""
    for first in (0, 1, 8):
        d = conv_inputs(dtype, (2, 45, 64), 4, None, True, False, seed=5)
        c = cuda(d)
        wide = torch.full((2, 45, 200), float("nan"), dtype=dtype, device="cuda")
        x = wide[..., first:first + 64]
        x.copy_(c["x"])
        y, _ = pkg.short_conv(x, c["weight"], c["bias"], silu=True)
        plain, _ = pkg.short_conv(c["x"], c["weight"], c["bias"], silu=True)
        assert torch.equal(y, plain)
        out = wide.new_zeros(2, 45, 100)[..., 3:67]
        pkg.short_conv(x, c["weight"], c["bias"], silu=True, out=out)
        assert torch.equal(out, plain)
        g = pkg.short_conv_grad(c["dy"], x, c["weight"], c["bias"], silu=True)
        h = pkg.short_conv_grad(c["dy"], c["x"], c["weight"], c["bias"], silu=True)
        close(g.x, h.x.cpu().double())
        close(g.weight, h.weight.cpu().double())
        # batch and rows the other way round
        xt = c["x"].transpose(0, 1).contiguous().transpose(0, 1)
        assert torch.equal(pkg.short_conv(xt, c["weight"], c["bias"], silu=True)[0], plain)


def test_conv_keeps_sequences_apart(pkg):
    """NaN and infinities of one packed sequence reach no other."""
    d = cuda(conv_inputs(torch.float32, (97, 40), 4, "mixed", True, True))
    o = d["offsets"].tolist()
    plain = pkg.short_conv(d["x"], d["weight"], d["bias"], state=d["state"], offsets=d["offsets"])
    x = d["x"].clone()
    x[o[1]:o[2]] = float("nan")
    x[o[0]] = float("inf")
    got = pkg.short_conv(x, d["weight"], d["bias"], state=d["state"], offsets=d["offsets"])
    assert torch.equal(got[0][o[2]:], plain[0][o[2]:])
    assert torch.equal(got[1][2:], plain[1][2:])


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("width", [1, 2, 4, 8])
@pytest.mark.parametrize("batch,ch", [(1, 64), (5, 33), (64, 128)])
def test_conv_steps_continue_a_prompt(pkg, dtype, width, batch, ch):
    d = cuda(conv_inputs(dtype, (batch, 9, ch), width, None, True, False))
    y, last = pkg.short_conv(d["x"], d["weight"], d["bias"], silu=True)
    slots = torch.randperm(batch + 3, generator=torch.Generator().manual_seed(1))[:batch]
    slots = slots.to(torch.int32).cuda()
    cache = torch.full((batch + 3, width - 1, ch), 7.0, dtype=dtype, device="cuda")
    _, first = pkg.short_conv(d["x"][:, :4], d["weight"], d["bias"], silu=True)
    cache[slots.long()] = first
    for t in range(4, 9):
        yt = pkg.short_conv_step(d["x"][:, t], cache, d["weight"], d["bias"], silu=True,
                                 slots=slots)
        close(yt, y[:, t].cpu().double())
    assert torch.equal(cache[slots.long()], last)
    rest = torch.ones(batch + 3, dtype=torch.bool, device="cuda")
    rest[slots.long()] = False
    assert (cache[rest] == 7).all()


def test_steps_outside_the_cache(pkg):
    d = cuda(conv_inputs(torch.float32, (4, 1, 32), 4, None, True, False))
    cache = torch.randn(3, 3, 32, device="cuda")
    before = cache.clone()
    slots = torch.tensor([-1, 2, 3, 2 ** 31 - 1], dtype=torch.int32, device="cuda")
    y = pkg.short_conv_step(d["x"][:, 0], cache, d["weight"], d["bias"], slots=slots)
    assert (y[[0, 2, 3]] == 0).all() and (y[1] != 0).any()
    assert torch.equal(cache[:2], before[:2]) and not torch.equal(cache[2], before[2])
    s = cuda(scan_inputs(torch.float32, (4, 1, 32), 16, 1, None))
    cache = torch.randn(3, 32, 16, device="cuda")
    before = cache.clone()
    y = pkg.state_scan_step(s["u"][:, 0], s["dt"][:, 0], s["A"], s["B"][:, 0], s["C"][:, 0],
                            cache, softplus=True, slots=slots)
    assert (y[[0, 2, 3]] == 0).all() and (y[1] != 0).any()
    assert torch.equal(cache[:2], before[:2]) and not torch.equal(cache[2], before[2])


# --------------------------------------------------------------------- scan
def scan_inputs(dtype, shape, n, groups, packed, seed=0, options=True, plus=True):
    gen = torch.Generator().manual_seed(seed)
    ch = shape[-1]
    off = offsets_of(packed_lengths(shape[0], packed)) if packed else None
    seqs = len(off) - 1 if packed else shape[0]
    lead = shape[:-1]
    d = {"u": randn(gen, *shape, dtype=dtype), "dt": randn(gen, *shape, dtype=dtype, scale=0.5),
         "A": -torch.arange(1, n + 1).float() * torch.exp(randn(gen, ch, n, scale=0.2)),
         "B": randn(gen, *lead, groups, n, dtype=dtype),
         "C": randn(gen, *lead, groups, n, dtype=dtype),
         "skip": None, "gate": None, "dt_bias": None, "state": None}
    if not plus:
        d["dt"] = (d["dt"].float().abs() * 0.2).to(dtype)
    if options:
        d.update(skip=randn(gen, ch), gate=randn(gen, *shape, dtype=dtype),
                 dt_bias=randn(gen, ch, scale=0.5) - 3, state=randn(gen, seqs, ch, n))
    d["offsets"] = off
    d["dy"] = randn(gen, *shape, dtype=dtype)
    d["dlast"] = randn(gen, seqs, ch, n)
    return d


SCAN = ("u", "dt", "A", "B", "C", "skip", "gate", "dt_bias", "state")


def check_scan(pkg, d, plus=True, dlast=True):
    c = cuda(d)
    args = [c[k] for k in SCAN[:5]]
    more = {k: c[k] for k in SCAN[5:] + ("offsets",)}
    y, last, marks = pkg.state_scan(*args, softplus=plus, marks=True, **more)
    y2, last2 = pkg.state_scan(*args, softplus=plus, **more)
    assert torch.equal(y, y2) and torch.equal(last, last2)
    g = pkg.state_scan_grad(c["dy"], *args, softplus=plus, marks=marks,
                            dlast=c["dlast"] if dlast else None, **more)
    leaf = {k: d[k].double().requires_grad_() if d[k] is not None else None for k in SCAN}
    ry, rl = ref.scan(leaf["u"], leaf["dt"], leaf["A"], leaf["B"], leaf["C"], leaf["skip"],
                      leaf["gate"], leaf["dt_bias"], plus, leaf["state"], d["offsets"])
    close(y, ry, "y")
    close(last, rl, "last")
    names = [k for k in SCAN if leaf[k] is not None]
    loss = (ry * d["dy"].double()).sum()
    if dlast:
        loss = loss + (rl * d["dlast"].double()).sum()
    if not loss.requires_grad:
        loss = loss + sum(leaf[k].sum() * 0 for k in names)
    grads = torch.autograd.grad(loss, [leaf[k] for k in names], allow_unused=True)
    for k, w in zip(names, grads):
        close(getattr(g, k), w if w is not None else torch.zeros_like(leaf[k]), "d" + k)
    for k in SCAN[5:]:
        assert (getattr(g, k) is None) == (d[k] is None)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("shape,n,groups,packed", [
    ((2, 37, 48), 16, 1, None), ((1, 1, 16), 16, 1, None), ((2, 2, 33), 16, 1, None),
    ((2, 70, 6), 1, 2, None), ((1, 33, 130), 4, 1, None), ((1, 65, 40), 7, 1, None),
    ((2, 40, 36), 13, 3, None), ((1, 64, 24), 32, 2, None), ((1, 45, 20), 64, 1, None),
    ((1, 34, 12), 100, 1, None), ((1, 40, 8), 128, 2, None), ((1, 300, 72), 16, 1, None),
    ((97, 40), 16, 1, "mixed"), ((60, 18), 16, 2, "empties"), ((50, 24), 8, 1, "singles"),
    ((64, 20), 5, 1, "one"), ((290, 36), 16, 1, "mixed"), ((96, 12), 33, 1, "mixed")])
def test_scan(pkg, dtype, shape, n, groups, packed):
    check_scan(pkg, scan_inputs(dtype, shape, n, groups, packed))


@pytest.mark.parametrize("left_out", SCAN[5:] + ("none", "all"))
@pytest.mark.parametrize("packed", [None, "mixed"])
@pytest.mark.parametrize("plus", [True, False])
def test_scan_options(pkg, left_out, packed, plus):
    shape = (83, 24) if packed else (2, 41, 24)
    d = scan_inputs(torch.float32, shape, 16, 1, packed, seed=2, options=left_out != "all",
                    plus=plus)
    if left_out in d:
        d[left_out] = None
    if not plus:
        d["dt_bias"] = None
    check_scan(pkg, d, plus, dlast=left_out != "all")


@pytest.mark.parametrize("packed", [None, "empties"])
def test_scan_of_no_rows(pkg, packed):
    d = scan_inputs(torch.float32, (0, 24) if packed else (2, 0, 24), 16, 1, packed)
    check_scan(pkg, d)


def test_scan_without_sequences(pkg):
    d = cuda(scan_inputs(torch.float32, (0, 5, 24), 16, 1, None))
    y, last, marks = pkg.state_scan(*[d[k] for k in SCAN[:5]], marks=True)
    assert y.shape == (0, 5, 24) and last.shape == (0, 24, 16)
    g = pkg.state_scan_grad(d["dy"], *[d[k] for k in SCAN[:5]], marks=marks)
    assert (g.A == 0).all()


def test_scan_of_slices(pkg):
    """u, dt, gate, B and C inside wider projections, batch and rows swapped."""
    d = scan_inputs(torch.bfloat16, (3, 45, 32), 16, 2, None, seed=5)
    c = cuda(d)
    args, more = [c[k] for k in SCAN[:5]], {k: c[k] for k in SCAN[5:]}
    plain = pkg.state_scan(*args, softplus=True, marks=True, **more)
    want = pkg.state_scan_grad(c["dy"], *args, softplus=True, marks=plain[2], **more)

    def inside(t, first):
        flat = t.reshape(3, 45, -1).transpose(0, 1)
        wide = torch.full((45, 3, flat.shape[-1] + 21), float("nan"), dtype=t.dtype, device="cuda")
        part = wide[..., first:first + flat.shape[-1]]
        part.copy_(flat)
        part = part.transpose(0, 1)
        return part if t.dim() == 3 else part.unflatten(-1, t.shape[2:])

    for first in (0, 5, 8):
        moved = [inside(c["u"], first), inside(c["dt"], first), c["A"], inside(c["B"], first),
                 inside(c["C"], first)]
        opts = dict(more, gate=inside(c["gate"], first))
        got = pkg.state_scan(*moved, softplus=True, marks=True, **opts)
        for a, b in zip(got, plain):
            assert torch.equal(a, b)
        g = pkg.state_scan_grad(inside(c["dy"], first), *moved, softplus=True, marks=got[2], **opts)
        for a, b in zip(g, want):
            assert torch.equal(a, b)
    # one row of B and C broadcast over the batch
    one = [c["u"], c["dt"], c["A"], c["B"][:1].expand(3, -1, -1, -1),
           c["C"][:1].expand(3, -1, -1, -1)]
    same = [c["u"], c["dt"], c["A"], one[3].contiguous(), one[4].contiguous()]
    assert torch.equal(pkg.state_scan(*one, softplus=True)[0],
                       pkg.state_scan(*same, softplus=True)[0])


def test_scan_keeps_sequences_apart(pkg):
    """NaN and infinities of one packed sequence reach no other, either way."""
    d = cuda(scan_inputs(torch.float32, (290, 36), 16, 1, "mixed"))
    o = d["offsets"].tolist()
    args, more = [d[k] for k in SCAN[:5]], {k: d[k] for k in SCAN[5:] + ("offsets",)}
    y, last, marks = pkg.state_scan(*args, softplus=True, marks=True, **more)
    g = pkg.state_scan_grad(d["dy"], *args, softplus=True, marks=marks, **more)
    u = d["u"].clone()
    u[o[2]:o[3]] = float("nan")
    u[o[3]] = float("inf")
    args[0] = u
    y2, last2, marks2 = pkg.state_scan(*args, softplus=True, marks=True, **more)
    g2 = pkg.state_scan_grad(d["dy"], *args, softplus=True, marks=marks2, **more)
    keep = torch.ones(290, dtype=torch.bool, device="cuda")
    keep[o[2]:o[4]] = False
    assert torch.equal(y2[keep], y[keep]) and not torch.isfinite(y2[~keep]).any(-1).all()
    keep_s = torch.ones(len(o) - 1, dtype=torch.bool, device="cuda")
    keep_s[2:4] = False
    assert torch.equal(last2[keep_s], last[keep_s])
    for k in ("u", "dt", "gate", "B"):
        assert torch.equal(getattr(g2, k)[keep], getattr(g, k)[keep]), k
    assert torch.equal(g2.state[keep_s], g.state[keep_s])


@pytest.mark.parametrize("shape,packed", [((1, 4096, 8), None), ((1, 2500, 40), None),
                                          ((5000, 8), "mixed")])
def test_long_scan_in_chunks(pkg, shape, packed):
    """Few channels and many rows: the rows are split, and the states carried,
    also where sequences open at and within the parts.  The reference runs the
    same sequences in 64 bits on the GPU, all channels of a row at once."""
    d = scan_inputs(torch.float32, shape, 16, 1, packed, seed=7)
    c = cuda(d)
    args, more = [c[k] for k in SCAN[:5]], {k: c[k] for k in SCAN[5:] + ("offsets",)}
    y, last, marks = pkg.state_scan(*args, softplus=True, marks=True, **more)
    g = pkg.state_scan_grad(c["dy"], *args, softplus=True, marks=marks, dlast=c["dlast"], **more)
    leaf = {k: d[k].double().requires_grad_() for k in SCAN}
    ry, rl = ref.scan(leaf["u"], leaf["dt"], leaf["A"], leaf["B"], leaf["C"], leaf["skip"],
                      leaf["gate"], leaf["dt_bias"], True, leaf["state"], d["offsets"])
    close(y, ry, "y")
    close(last, rl, "last")
    loss = (ry * d["dy"].double()).sum() + (rl * d["dlast"].double()).sum()
    for k, w in zip(SCAN, torch.autograd.grad(loss, [leaf[k] for k in SCAN])):
        close(getattr(g, k), w, "d" + k)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("n,groups", [(1, 1), (5, 1), (16, 1), (16, 2), (64, 1), (128, 4)])
@pytest.mark.parametrize("batch,ch", [(1, 64), (5, 36), (33, 128)])
def test_scan_steps_continue_a_prompt(pkg, dtype, n, groups, batch, ch):
    d = scan_inputs(dtype, (batch, 8, ch), n, groups, None)
    c = cuda(d)
    ry, rl = ref.scan(*[d[k].double() for k in SCAN[:5]], d["skip"].double(), d["gate"].double(),
                      d["dt_bias"].double(), True)
    gen = torch.Generator().manual_seed(1)
    slots = torch.randperm(batch + 3, generator=gen)[:batch].to(torch.int32).cuda()
    cache = torch.full((batch + 3, ch, n), 7.0, device="cuda")
    cut = lambda v, s: v[:, s] if v.dim() > 2 else v  # noqa: E731
    _, cache[slots.long()] = pkg.state_scan(
        *[cut(c[k], slice(0, 3)) for k in SCAN[:5]], skip=c["skip"], gate=c["gate"][:, :3],
        dt_bias=c["dt_bias"], softplus=True)
    for t in range(3, 8):
        yt = pkg.state_scan_step(*[cut(c[k], t) for k in SCAN[:5]], cache, skip=c["skip"],
                                 gate=c["gate"][:, t], dt_bias=c["dt_bias"], softplus=True,
                                 slots=slots)
        close(yt, ry[:, t])
    close(cache[slots.long()], rl)
    rest = torch.ones(batch + 3, dtype=torch.bool, device="cuda")
    rest[slots.long()] = False
    assert (cache[rest] == 7).all()


def test_extreme_step_sizes(pkg):
    """Decays that vanish and that do nothing: exp(-inf) = 0 and exp(0) = 1."""
    d = scan_inputs(torch.float32, (1, 40, 8), 16, 1, None, plus=False)
    d["dt"][:, 3::7] = 300.0
    d["dt"][:, 4::7] = 0.0
    d["dt"][:, 5::7] = 1e30
    d["u"][:, 5::7] = 0.0
    d["dt_bias"] = None
    c = cuda(d)
    more = {k: c[k] for k in SCAN[5:]}
    y, last = pkg.state_scan(*[c[k] for k in SCAN[:5]], **more)
    leaf = {k: d[k].double() if d[k] is not None else None for k in SCAN}
    ry, rl = ref.scan(*[leaf[k] for k in SCAN[:5]], leaf["skip"], leaf["gate"], None, False,
                      leaf["state"])
    close(y, ry)
    close(last, rl)
    # softplus of what overflows exp and of what underflows
    d["dt"] = torch.tensor([-1e4, -100.0, -20.0, 0.0, 20.0, 88.0, 200.0, 1e4]).repeat(1, 40, 1)
    c = cuda(d)
    y, last = pkg.state_scan(*[c[k] for k in SCAN[:5]], softplus=True, **more)
    ry, rl = ref.scan(d["u"].double(), d["dt"].double(), *[leaf[k] for k in SCAN[2:5]],
                      leaf["skip"], leaf["gate"], None, True, leaf["state"])
    close(y, ry)
    close(last, rl)


def test_gradients_against_differences(pkg):
    """The kernels' gradients along a random direction against central
    differences of the definition in 64 bits (step 1e-5: truncation 1e-10)."""
    d = scan_inputs(torch.float32, (2, 37, 12), 16, 1, None, seed=11)
    c = cuda(d)
    args, more = [c[k] for k in SCAN[:5]], {k: c[k] for k in SCAN[5:]}
    _, _, marks = pkg.state_scan(*args, softplus=True, marks=True, **more)
    g = pkg.state_scan_grad(c["dy"], *args, softplus=True, marks=marks, dlast=c["dlast"], **more)
    gen = torch.Generator().manual_seed(4)

    def loss(v):
        y, last = ref.scan(*[v[k] for k in SCAN[:8]], True, v["state"])
        return (y * d["dy"].double()).sum() + (last * d["dlast"].double()).sum()

    for k in SCAN:
        base = {n: d[n].double() for n in SCAN}
        way = torch.randn(d[k].shape, generator=gen, dtype=torch.float64)
        up, down = dict(base), dict(base)
        up[k], down[k] = base[k] + 1e-5 * way, base[k] - 1e-5 * way
        want = float((loss(up) - loss(down)) / 2e-5)
        got = float((getattr(g, k).cpu().double() * way).sum())
        scale = float(getattr(g, k).cpu().double().norm())
        assert abs(got - want) <= 1e-4 * scale, k
    d = conv_inputs(torch.float32, (2, 19, 12), 4, None, True, True, seed=12)
    c = cuda(d)
    g = pkg.short_conv_grad(c["dy"], c["x"], c["weight"], c["bias"], silu=True, state=c["state"],
                            dlast=c["dlast"])

    def loss(v):
        y, last = ref.conv(v["x"], v["weight"], v["bias"], True, v["state"])
        return (y * d["dy"].double()).sum() + (last * d["dlast"].double()).sum()

    for k in ("x", "weight", "bias", "state"):
        base = {n: d[n].double() for n in ("x", "weight", "bias", "state")}
        way = torch.randn(d[k].shape, generator=gen, dtype=torch.float64)
        up, down = dict(base), dict(base)
        up[k], down[k] = base[k] + 1e-5 * way, base[k] - 1e-5 * way
        want = float((loss(up) - loss(down)) / 2e-5)
        got = float((getattr(g, k).cpu().double() * way).sum())
        assert abs(got - want) <= 1e-4 * float(getattr(g, k).cpu().double().norm()), k


def test_autograd(pkg):
    """The differentiable calls give what the gradient calls give."""
    d = cuda(scan_inputs(torch.float32, (2, 37, 24), 16, 1, None, seed=3))
    leaf = {k: d[k].clone().requires_grad_() for k in SCAN}
    y, last = pkg.state_scan(*[leaf[k] for k in SCAN[:5]], softplus=True,
                             **{k: leaf[k] for k in SCAN[5:]})
    ((y * d["dy"]).sum() + (last * d["dlast"]).sum()).backward()
    args, more = [d[k] for k in SCAN[:5]], {k: d[k] for k in SCAN[5:]}
    _, _, marks = pkg.state_scan(*args, softplus=True, marks=True, **more)
    g = pkg.state_scan_grad(d["dy"], *args, softplus=True, marks=marks, dlast=d["dlast"], **more)
    for k in SCAN:
        assert torch.equal(leaf[k].grad, getattr(g, k)), k
    c = cuda(conv_inputs(torch.float32, (2, 37, 24), 4, None, True, True))
    leaf = {k: c[k].clone().requires_grad_() for k in ("x", "weight", "bias", "state")}
    y, last = pkg.short_conv(leaf["x"], leaf["weight"], leaf["bias"], silu=True,
                             state=leaf["state"])
    (y * c["dy"]).sum().backward()  # last unused: its gradient is zeros
    g = pkg.short_conv_grad(c["dy"], c["x"], c["weight"], c["bias"], silu=True, state=c["state"])
    for k in leaf:
        assert torch.equal(leaf[k].grad, getattr(g, k)), k


def test_streams_graphs_and_repeats(pkg):
    """Another stream, a captured graph and a second run give the same bits."""
    d = cuda(scan_inputs(torch.bfloat16, (1, 700, 40), 16, 1, None, seed=9))
    args, more = [d[k] for k in SCAN[:5]], {k: d[k] for k in SCAN[5:]}

    def both(stream=None):
        y, last, marks = pkg.state_scan(*args, softplus=True, marks=True, stream=stream, **more)
        g = pkg.state_scan_grad(d["dy"], *args, softplus=True, marks=marks, stream=stream, **more)
        return [y, last] + list(g)

    want = both()
    torch.cuda.synchronize()
    for a, b in zip(both(), want):
        assert torch.equal(a, b)
    s = torch.cuda.Stream()
    got = both(s)
    s.synchronize()
    for a, b in zip(got, want):
        assert torch.equal(a, b)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = both()
    graph.replay()
    torch.cuda.synchronize()
    for a, b in zip(got, want):
        assert torch.equal(a, b)


def test_refusals(pkg):
    d = cuda(scan_inputs(torch.float32, (2, 5, 24), 16, 2, None))
    ok = {k: d[k] for k in SCAN}

    def scan(**change):
        v = dict(ok, **change)
        return pkg.state_scan(*[v.pop(k) for k in SCAN[:5]], **v)

    scan()
    bad = [dict(u=d["u"].cpu()), dict(u=d["u"].double()), dict(dt=d["dt"].bfloat16()),
           dict(dt=d["dt"][:, :4]), dict(A=d["A"].T), dict(A=d["A"].half()), dict(B=d["B"][..., :8]),
           dict(B=d["B"].transpose(-1, -2)), dict(u=d["u"].transpose(1, 2)),
           dict(state=d["state"][:1]), dict(state=d["state"].bfloat16()), dict(skip=d["skip"][:5]),
           dict(offsets=torch.tensor([0, 10], device="cuda", dtype=torch.int32)),
           dict(B=torch.zeros(2, 5, 5, 16, device="cuda"), C=torch.zeros(2, 5, 5, 16, device="cuda")),
           dict(B=torch.zeros(2, 5, 1, 129, device="cuda"), C=torch.zeros(2, 5, 1, 129, device="cuda"))]
    for change in bad:
        with pytest.raises((TypeError, ValueError)):
            scan(**change)
    with pytest.raises(ValueError):
        pkg.state_scan_grad(d["dy"], *[d[k] for k in SCAN[:5]],
                            marks=torch.zeros(1, device="cuda"))
    c = cuda(conv_inputs(torch.float32, (2, 5, 24), 4, None, True, True))
    for change in (dict(x=c["x"].cpu()), dict(x=c["x"].int()), dict(weight=c["weight"].half()),
                   dict(weight=torch.zeros(24, 9, device="cuda")), dict(bias=c["bias"][:3]),
                   dict(state=c["state"][:, :2]), dict(x=c["x"].transpose(1, 2)), dict(x=None)):
        v = dict(x=c["x"], weight=c["weight"], bias=c["bias"], state=c["state"], **{})
        v.update(change)
        with pytest.raises((TypeError, ValueError)):
            pkg.short_conv(v["x"], v["weight"], v["bias"], state=v["state"])
    with pytest.raises(ValueError):
        pkg.short_conv_step(c["x"][:, 0], c["state"][:1], c["weight"])
    with pytest.raises(ValueError):
        pkg.short_conv_step(c["x"][:, 0].requires_grad_(), c["state"], c["weight"])
    packed = torch.zeros(10, 24, device="cuda")
    for off in (torch.tensor([0, 10], device="cuda"), torch.tensor([0, 10], dtype=torch.int32),
                torch.zeros(0, dtype=torch.int32, device="cuda")):
        with pytest.raises(ValueError):
            pkg.short_conv(packed, c["weight"], offsets=off)


def test_offsets_out_of_order_stay_in_range(pkg):
    """Offsets that break their contract give some result within the tensors:
    the guard values around the outputs stay."""
    d = cuda(scan_inputs(torch.float32, (70, 24), 16, 1, "mixed"))
    c = cuda(conv_inputs(torch.float32, (70, 24), 4, "mixed", True, False))
    n = d["offsets"].shape[0]
    for off in ([50, 10] * n, [-5, 200] * n, [0] * n, [70] * n):
        off = torch.tensor(off[:n], dtype=torch.int32, device="cuda")
        buf = torch.full((90, 24), 9.0, device="cuda")
        pkg.state_scan(*[d[k] for k in SCAN[:5]], softplus=True, offsets=off, out=buf[10:80])
        assert (buf[:10] == 9).all() and (buf[80:] == 9).all()
        buf.fill_(9.0)
        pkg.short_conv(c["x"], c["weight"], offsets=off, out=buf[10:80])
        assert (buf[:10] == 9).all() and (buf[80:] == 9).all()
    torch.cuda.synchronize()


def test_no_step_leaves_the_state(pkg):
    """d = 0 is a decay of exactly 1 and no input: the bits of the state stay,
    over prompts (whole and in parts) and tokens."""
    for rows in (40, 5000):
        d = cuda(scan_inputs(torch.float32, (1, rows, 8), 16, 1, None))
        zero = torch.zeros_like(d["dt"])
        y, last = pkg.state_scan(d["u"], zero, d["A"], d["B"], d["C"], state=d["state"])
        assert torch.equal(last, d["state"])
        want = torch.einsum("cn,rn->rc", d["state"][0].double(), d["C"][0, :, 0].double())
        close(y[0], want.cpu())
    cache = d["state"].clone()
    pkg.state_scan_step(d["u"][:, 0], zero[:, 0], d["A"], d["B"][:, 0], d["C"][:, 0], cache)
    assert torch.equal(cache, d["state"])


def test_outputs_over_inputs_are_refused(pkg):
    d = cuda(scan_inputs(torch.float32, (2, 37, 24), 16, 1, None))
    args = [d[k] for k in SCAN[:5]]
    w = torch.randn(24, 4, device="cuda")
    for out in (d["u"], d["dt"]):
        with pytest.raises(ValueError):
            pkg.state_scan(*args, out=out)
    with pytest.raises(ValueError):
        pkg.short_conv(d["u"], w, out=d["u"])
    wide = torch.randn(2, 37, 64, device="cuda")
    with pytest.raises(ValueError):
        pkg.short_conv(wide[..., :24], w, out=wide[..., 20:44])
    want = pkg.short_conv(wide[..., :24].clone(), w)[0]
    pkg.short_conv(wide[..., :24], w, out=wide[..., 24:48])
    assert torch.equal(wide[..., 24:48], want)
    # a gradient is recorded on the current stream, for outputs of the call's own
    u = d["u"].clone().requires_grad_()
    for more in ({"out": torch.empty_like(d["u"])}, {"stream": torch.cuda.Stream()}):
        with pytest.raises(ValueError):
            pkg.short_conv(u, w, **more)
        with pytest.raises(ValueError):
            pkg.state_scan(u, *args[1:], **more)


def test_gradients_beside_other_streams(pkg):
    """Backward passes under a stream that is not the default one."""
    c = cuda(conv_inputs(torch.float32, (2, 300, 64), 4, None, True, False))
    want = pkg.short_conv_grad(c["dy"], c["x"], c["weight"], c["bias"], silu=True)
    torch.cuda.synchronize()
    s = torch.cuda.Stream()
    with torch.cuda.stream(s):
        x = c["x"].clone().requires_grad_()
        y, _ = pkg.short_conv(x, c["weight"], c["bias"], silu=True)
        (y * c["dy"]).sum().backward()
    s.synchronize()
    assert torch.equal(x.grad, want.x)


def test_offsets_beyond_32_bits(pkg):
    """Tensors of more than 2^31 elements: the last channels of the last rows,
    and the last entries of a cache, as they are in small tensors."""
    rows, ch = 70016, 32768
    assert rows * ch > 2 ** 31
    gen = torch.Generator(device="cuda").manual_seed(3)
    u = torch.empty(1, rows, ch, dtype=torch.bfloat16, device="cuda").normal_(generator=gen)
    w = torch.randn(ch, 4, generator=gen, device="cuda")
    y, last = pkg.short_conv(u, w, silu=True)
    part = u[..., -64:].contiguous()
    want, want_last = pkg.short_conv(part, w[-64:].contiguous(), silu=True)
    assert torch.equal(y[..., -64:], want) and torch.equal(last[..., -64:], want_last)
    g = pkg.short_conv_grad(y, u, w, silu=True)
    h = pkg.short_conv_grad(want, part, w[-64:].contiguous(), silu=True)
    close(g.x[:, -300:, -64:], h.x[:, -300:].cpu().double())
    close(g.weight[-64:], h.weight.cpu().double())
    del g, y
    A = -torch.rand(ch, 2, generator=gen, device="cuda") - 0.5
    B, C = (torch.randn(1, rows, 2, generator=gen, device="cuda").bfloat16() for _ in range(2))
    y, last = pkg.state_scan(u, u, A, B, C, softplus=True)
    want, want_last = pkg.state_scan(part, part, A[-64:].contiguous(), B, C, softplus=True)
    close(y[:, -300:, -64:], want[:, -300:].cpu().double())
    close(last[:, -64:], want_last.cpu().double())
    del u, y
    entries, ch, n = 140000, 1024, 16
    assert entries * ch * n > 2 ** 31
    cache = torch.zeros(entries, ch, n, device="cuda")
    small = torch.zeros(2, ch, n, device="cuda")
    s = cuda(scan_inputs(torch.float32, (2, 1, ch), n, 1, None))
    args = [s[k][:, 0] if s[k].dim() > 2 else s[k] for k in SCAN[:5]]
    slots = torch.tensor([entries - 1, entries - 2], dtype=torch.int32, device="cuda")
    for _ in range(2):
        got = pkg.state_scan_step(*args, cache, softplus=True, slots=slots)
        want = pkg.state_scan_step(*args, small, softplus=True)
        assert torch.equal(got, want)
    assert torch.equal(cache[slots.long()], small) and not cache[:-2].any()
