"""The branches of the sequence operators that only large or long calls take,
against 64 bits: rows split over the card with several batch entries and
groups, at every number of lanes a channel has; several entries of a token
call in one thread; convolution runs of more than one block of rows.
Tolerances are test_sequence.py's."""
import pytest
import torch

import sequence_reference as ref
from test_sequence import SCAN, TYPES, check_scan, close, cuda, offsets_of, randn, scan_inputs

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def pkg():
    from paper_1908_06649_gb300 import _build
    _build.build()
    import paper_1908_06649_gb300 as p
    p.lib()
    return p


def sms():
    return torch.cuda.get_device_properties(0).multi_processor_count


# ------------------------------------------------------- rows over the card
@pytest.mark.parametrize("dtype,n,groups,per_group,packed", [
    (torch.float32, 4, 2, 8, None), (torch.float32, 4, 3, 5, "mixed"),
    (torch.float32, 13, 3, 5, None), (torch.bfloat16, 16, 3, 8, "mixed"),
    (torch.float32, 16, 2, 40, None), (torch.float32, 32, 2, 8, None),
    (torch.float16, 32, 2, 8, "mixed"), (torch.float32, 29, 2, 3, "mixed"),
    (torch.float32, 64, 2, 8, None), (torch.bfloat16, 64, 1, 24, "mixed"),
    (torch.float32, 64, 3, 3, None), (torch.float32, 128, 2, 8, None),
    (torch.float16, 128, 2, 8, "mixed"), (torch.float32, 121, 2, 3, "empties")])
def test_split_rows(pkg, dtype, n, groups, per_group, packed):
    """Forward from 6 and gradient from 4 tiles of 32 rows on, where few blocks
    leave the card empty; in words (channels of a group a multiple of 8) and
    value by value."""
    lead = (331,) if packed else (2, 215)
    d = scan_inputs(dtype, lead + (groups * per_group,), n, groups, packed, seed=n)
    check_scan(pkg, d)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("n", [8, 32, 64, 128])
def test_words_of_rows_at_every_state_count(pkg, dtype, n):
    """Rows in words, whole: few enough rows not to be split."""
    check_scan(pkg, scan_inputs(dtype, (2, 53, 48), n, 2, None, seed=n))


# ------------------------------------------- several entries in one thread
@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("n,groups", [(5, 1), (8, 2), (13, 1), (16, 4), (32, 1), (61, 1), (128, 2)])
def test_token_entries_together(pkg, dtype, n, groups):
    """Enough threads for several entries each (2 where two lanes share a
    channel, else 4), the last group of entries not full, with entries outside the
    cache among the others; cache and outputs against 64 bits."""
    lanes = 2
    while lanes * 4 < n:
        lanes *= 2
    together = 2 if lanes == 2 else 4
    ch = 364
    batch = -(-together * 1024 * sms() // (lanes * ch)) // together * together + together + 1
    assert ch * batch * lanes >= together * 1024 * sms() and batch % together
    d = cuda(scan_inputs(dtype, (batch, 1, ch), n, groups, None, seed=n))
    gen = torch.Generator().manual_seed(n)
    entries = batch + 5
    slots = torch.randperm(entries, generator=gen)[:batch].to(torch.int32)
    dead = torch.rand(batch, generator=gen) < 0.2
    dead[-1], dead[-2] = True, False
    slots[dead] = torch.tensor([-1, entries, 2 ** 31 - 1] * batch, dtype=torch.int32)[:int(dead.sum())]
    slots, dead = slots.cuda(), dead.cuda()
    cache = torch.randn(entries, ch, n, generator=gen).cuda()
    before = cache.clone()
    one = {k: d[k][:, 0] if k in ("u", "dt", "B", "C", "gate") else d[k] for k in SCAN[:8]}
    args, more = [one[k] for k in SCAN[:5]], {k: one[k] for k in SCAN[5:8]}
    y = pkg.state_scan_step(*args, cache, slots=slots, softplus=True, **more)
    f = {k: v.double() for k, v in one.items()}
    at = slots[~dead].long()
    step = ref.softplus(f["dt"] + f["dt_bias"])
    B, C = (f[k].repeat_interleave(ch // groups, 1) for k in ("B", "C"))
    h = before[at].double() * torch.exp(step[..., None] * f["A"])[~dead]
    h = h + ((step * f["u"])[..., None] * B)[~dead]
    o = (h * C[~dead]).sum(-1) + (f["skip"] * f["u"])[~dead]
    close(y[~dead], (o * ref.silu(f["gate"])[~dead]).cpu(), "y")
    close(cache[at], h.cpu(), "state")
    assert (y[dead] == 0).all()
    rest = torch.ones(entries, dtype=torch.bool, device="cuda")
    rest[at] = False
    assert torch.equal(cache[rest], before[rest])


# --------------------------------------------------- long convolution runs
def conv64(x, w, bias, state, offsets):
    """The convolution with silu in 64 bits on the GPU, all rows at once."""
    rows, (ch, width) = torch.arange(x.shape[0], device="cuda"), w.shape
    off = offsets.long()
    seq = torch.searchsorted(off[1:].contiguous(), rows, right=True)
    # every sequence behind its past in one array
    first = off[:-1] + (width - 1) * torch.arange(len(off) - 1, device="cuda")
    here = rows + (seq + 1) * (width - 1)
    past = (first[:, None] + torch.arange(width - 1, device="cuda")).flatten()
    ends = (past.view(len(off) - 1, width - 1) + (off[1:] - off[:-1])[:, None]).flatten()
    padded = x.new_zeros(x.shape[0] + state.shape[0] * (width - 1), ch)
    padded = padded.index_copy(0, here, x).index_copy(0, past, state.reshape(-1, ch))
    p = bias.expand_as(x)
    for k in range(width):
        p = p + w[:, k] * padded[here - (width - 1) + k]
    return ref.silu(p), padded[ends].view(state.shape)


@pytest.mark.parametrize("dtype,width,ch,lengths", [
    (torch.float32, 3, 4099, [1500, 1, 0, 77, 2, 1003]), (torch.bfloat16, 5, 4096, [2000, 9, 991]),
    (torch.float16, 7, 4096, [6, 1700, 1, 1, 1400]), (torch.bfloat16, 4, 8192, [3, 1530, 0]),
    (torch.float32, 8, 2048, [5000, 400]), (torch.bfloat16, 2, 4097, [1, 3000]),
    (torch.float16, 1, 4096, [2700, 300]), (torch.float32, 6, 4096, [50] * 60)])
def test_long_convolution_runs(pkg, dtype, width, ch, lengths):
    """Runs of two and more blocks of 8 rows, which load ahead, over packed
    sequences that end anywhere in them."""
    rows = sum(lengths)
    assert rows * ch >= 2 * 1024 * sms() * 8 * 4  # values a thread: 4 forward, 2 in the gradient
    gen = torch.Generator().manual_seed(width)
    off = offsets_of(lengths).cuda()
    x, dy = (randn(gen, rows, ch, dtype=dtype).cuda() for _ in range(2))
    state, dlast = (randn(gen, len(lengths), width - 1, ch, dtype=dtype).cuda() for _ in range(2))
    w, bias = randn(gen, ch, width, scale=width ** -0.5).cuda(), randn(gen, ch, scale=0.3).cuda()
    y, last = pkg.short_conv(x, w, bias, silu=True, state=state, offsets=off)
    g = pkg.short_conv_grad(dy, x, w, bias, silu=True, state=state, offsets=off, dlast=dlast)
    leaf = [t.double().requires_grad_() for t in (x, w, bias, state)]
    ry, rl = conv64(*leaf, off)
    close(y, ry.cpu(), "y")
    close(last, rl.cpu(), "last")
    loss = (ry * dy.double()).sum() + (rl * dlast.double()).sum()
    for k, got, want in zip(("x", "weight", "bias", "state"), g, torch.autograd.grad(loss, leaf)):
        close(got, want.cpu(), "d" + k)
