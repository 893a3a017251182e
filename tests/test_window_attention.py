"""Window attention on the GPU against its definition in 64 bits
(mixing_reference.py): prompts, gradients, tokens from caches; and what it
refuses.

Tolerances, set before the first run, u half a step of the rows' type.  The
weights p are rounded to it, each by at most u of itself: with errors of random
sign the output is u of its norm off, the rounding of the output another u.
In the gradient ds is rounded so too, and delta is formed from the rounded y,
at most u of |dy||y| where dp is |dy||v| and |y| <= |v|: 3 u before the last
rounding.  Value by value, where rows of few keys are far larger than others, u
is taken of the sum of its terms' sizes instead, which bounds what their
roundings can do.  Products and sums in fp32 and exponentials of the special function
unit (2^-22, and 2^-23 of an argument below 2^6) add less than 2e-5."""
import pytest
import torch

import mixing_reference as ref
from mixing_reference import U, close, cuda, offsets_of, packed_lengths, randn

gpu = pytest.mark.gpu
HALF = [torch.bfloat16, torch.float16]


@pytest.fixture(scope="module")
def tcu():
    from paper_1908_06649_gb300 import _build
    _build.build()
    import paper_1908_06649_gb300 as p
    p.lib()
    return p


def inputs(dtype, lead, heads, kv, dim, seed=0, scale=1.0):
    gen = torch.Generator().manual_seed(seed)
    r = lambda h: randn(gen, *lead, h, dim, dtype=dtype, scale=scale)  # noqa: E731
    return dict(q=r(heads), k=r(kv), v=r(kv)), r(heads)


def check(tcu, a, dy, window, sinks, offsets=None, scale=None):
    u = U[dy.dtype]
    d = {n: t.double().requires_grad_() for n, t in a.items()}
    want, sums = ref.attention(**d, window=window, sinks=sinks, scale=scale, offsets=offsets)
    grads = torch.autograd.grad(want, list(d.values()), dy.double())
    more = dict(window=window, sinks=sinks, scale=scale,
                offsets=None if offsets is None else offsets.cuda())
    c = cuda(a)
    y, lse = tcu.window_attention(**c, **more, lse=True)
    close(y, want, "y", u + 2e-5)
    close(lse, sums, "lse")
    assert torch.equal(tcu.window_attention(**c, **more), y)
    g = tcu.window_attention_grad(dy.cuda(), **c, y=y, lse=lse, **more)
    with torch.no_grad():
        terms = ref.attention_terms(**d, dy=dy.double(), window=window, sinks=sinks, scale=scale,
                                    offsets=offsets)
    for n, got, exact, sizes in zip(g._fields, g, grads, terms):
        close(got, exact, "d" + n, 3 * u + 2e-5, sizes)
    for x, z in zip(g, tcu.window_attention_grad(dy.cuda(), **c, y=y, lse=lse, **more)):
        assert torch.equal(x, z)


@gpu
@pytest.mark.parametrize("dtype", HALF)
@pytest.mark.parametrize("batch,length,heads,kv,dim,window,sinks", [
    (1, 2, 1, 1, 64, 2, 0), (1, 128, 1, 1, 128, 128, 0), (1, 128, 2, 1, 64, 40, 0),
    (2, 130, 4, 2, 64, 50, 3), (1, 300, 4, 1, 128, 1000, 0), (2, 257, 3, 3, 80, 100, 5),
    (1, 600, 2, 2, 128, 33, 4), (1, 700, 2, 1, 64, 200, 150), (3, 65, 6, 2, 8, 7, 1),
    (1, 513, 8, 2, 128, 128, 130), (1, 400, 2, 1, 40, 1, 2), (2, 384, 5, 5, 96, 256, 0),
    (1, 200, 2, 2, 64, 2 ** 31 - 1, 2 ** 31 - 1)])
def test_dense(tcu, dtype, batch, length, heads, kv, dim, window, sinks):
    check(tcu, *inputs(dtype, (batch, length), heads, kv, dim), window, sinks)


@gpu
@pytest.mark.parametrize("dtype", HALF)
@pytest.mark.parametrize("kind", ["one", "empties", "singles", "mixed"])
@pytest.mark.parametrize("total,dim,window,sinks", [(77, 64, 20, 2), (700, 128, 90, 3), (650, 80, 1000, 0),
                                                    (1000, 64, 30, 70)])
def test_packed(tcu, dtype, kind, total, dim, window, sinks):
    off = offsets_of(packed_lengths(total, kind))
    check(tcu, *inputs(dtype, (total,), 4, 2, dim), window, sinks, offsets=off)


@gpu
@pytest.mark.parametrize("lengths,window,sinks", [
    ([2600], 100, 3), ([2100, 2500], 60, 3), ([700, 0, 1990, 50], 60, 130), ([100, 2300], 900, 4), ([1, 3000, 1], 30, 256),
    ([2500], 20, 300)])
def test_first_tokens_of_long_sequences(tcu, lengths, window, sinks):
    """Gradients of keys that thousands of rows see, which blocks of their own
    sum in part."""
    a, dy = inputs(torch.bfloat16, (sum(lengths),), 2, 1, 64)
    check(tcu, a, dy, window, sinks, offsets=offsets_of(lengths))
    if len(lengths) == 1:
        check(tcu, {n: t[None] for n, t in a.items()}, dy[None], window, sinks)


@gpu
@pytest.mark.parametrize("dtype", HALF)
def test_large_scores_and_scales(tcu, dtype):
    """Scores up to some hundreds: the running maximum rises again and again."""
    a, dy = inputs(dtype, (1, 400), 2, 1, 64)
    a["k"] *= torch.linspace(0.1, 8, 400)[:, None, None].to(dtype)
    check(tcu, a, dy, 300, 4)
    check(tcu, a, dy, 300, 4, scale=0.01)
    a["k"] = a["k"].flip(1)
    check(tcu, a, dy, 100, 4, scale=1.0)


@gpu
@pytest.mark.parametrize("dtype", HALF)
def test_a_window_of_one(tcu, dtype):
    """Every row sees itself alone: y is v, dv the sum over heads of dy, and dq
    and dk are what fp32 leaves of dp - delta, both some |dy||v|."""
    a, dy = inputs(dtype, (2, 150), 4, 2, 64)
    c, dy = cuda(a), dy.cuda()
    y, lse = tcu.window_attention(**c, window=1, lse=True)
    assert torch.equal(y, c["v"].repeat_interleave(2, 2))
    g = tcu.window_attention_grad(dy, **c, y=y, lse=lse, window=1)
    close(g.v, dy.double().unflatten(2, (2, 2)).sum(3).cpu(), inner=3 * U[dtype])
    size = 64 * dy.abs().max() * c["v"].abs().max() * max(c["q"].abs().max(), c["k"].abs().max()) / 8
    assert g.q.abs().max() <= 2e-6 * size and g.k.abs().max() <= 4e-6 * size


@gpu
@pytest.mark.parametrize("dtype", HALF)
def test_small_gradients(tcu, dtype):
    """Gradients near the bottom of fp16's range, of long rows of small weights,
    lose no more than others: dy is brought up before ds is rounded."""
    a, dy = inputs(dtype, (1, 600), 2, 1, 64)
    a = {n: t * 0.1 if n != "v" else t for n, t in a.items()}
    dy = (dy.float() * 2e-3).to(dtype)
    check(tcu, a, dy, 600, 0)


@gpu
@pytest.mark.parametrize("dtype", HALF)
def test_strides(tcu, dtype):
    """Slices of one projection, batch entries in another order."""
    gen = torch.Generator().manual_seed(3)
    big = randn(gen, 140, 2, 8 * 64 + 8, dtype=dtype).cuda().transpose(0, 1)
    q, k, v = (big[..., 8 + 64 * lo:8 + 64 * hi].unflatten(-1, (hi - lo, 64))
               for lo, hi in ((0, 4), (4, 6), (6, 8)))
    more = dict(window=60, sinks=2)
    y, lse = tcu.window_attention(q, k, v, lse=True, **more)
    flat = [t.contiguous() for t in (q, k, v)]
    y2, lse2 = tcu.window_attention(*flat, lse=True, **more)
    assert torch.equal(y, y2) and torch.equal(lse, lse2)
    g = tcu.window_attention_grad(q, q, k, v, q, lse, **more)
    w = tcu.window_attention_grad(flat[0], *flat, flat[0], lse, **more)
    for a, b in zip(g, w):
        assert torch.equal(a, b)
    out = torch.zeros(2, 140, 5, 64, dtype=dtype, device="cuda")
    tcu.window_attention(q, k, v, out=out[:, :, 1:], **more)
    assert torch.equal(out[:, :, 1:], y) and (out[:, :, 0] == 0).all()


@gpu
@pytest.mark.parametrize("dtype", HALF)
@pytest.mark.parametrize("used", [200, 256, 70])
def test_rows_behind_the_last_sequence(tcu, dtype, used):
    """Rows of no sequence that are no numbers: not read, not written, zero
    gradients."""
    nan = float("nan")
    a, dy = inputs(dtype, (300,), 4, 2, 80)
    off = offsets_of([60, 0, used - 60]).cuda()
    c, dy = cuda(a), dy.cuda()
    s = {n: t[:used].clone() for n, t in c.items()}
    for t in (*c.values(), dy):
        t[used:] = nan
    more = dict(window=50, sinks=3, offsets=off)
    out = torch.full_like(c["q"], 7)
    y, lse = tcu.window_attention(**c, lse=True, out=out, **more)
    y2, lse2 = tcu.window_attention(**s, lse=True, **more)
    assert torch.equal(out[:used], y2) and (out[used:] == 7).all() and torch.equal(lse[:used], lse2)
    y = y.clone()
    y[used:] = nan
    lse[used:] = nan
    g = tcu.window_attention_grad(dy, **c, y=y, lse=lse, **more)
    w = tcu.window_attention_grad(dy[:used].clone(), **s, y=y2, lse=lse2, **more)
    for got, want in zip(g, w):
        assert torch.equal(got[:used], want) and (got[used:] == 0).all()


@gpu
@pytest.mark.parametrize("dtype", HALF)
def test_batch_entries_do_not_reach_each_other(tcu, dtype):
    a, dy = inputs(dtype, (3, 70), 2, 1, 64)
    c, dy = cuda(a), dy.cuda()
    more = dict(window=20, sinks=1)
    y, lse = tcu.window_attention(**c, lse=True, **more)
    g = tcu.window_attention_grad(dy, **c, y=y, lse=lse, **more)
    for t in (*c.values(), dy):
        t[1] = float("nan")
    y2, lse2 = tcu.window_attention(**c, lse=True, **more)
    g2 = tcu.window_attention_grad(dy, **c, y=y2, lse=lse2, **more)
    for got, want in zip((y2, *g2), (y, *g)):
        assert torch.equal(got[::2], want[::2])


@gpu
@pytest.mark.parametrize("dtype", HALF)
@pytest.mark.parametrize("bad", [float("nan"), float("inf"), -float("inf")])
@pytest.mark.parametrize("where", [5, 63, 64, 200, 299])
def test_what_is_not_finite_reaches_who_sees_it(tcu, dtype, bad, where):
    """One row of k, v or q that is not finite, amid sequences that end inside
    tiles: rows that do not see it keep their results and gradients, and rows
    that see the value have no number."""
    a, dy = inputs(dtype, (300,), 4, 2, 80)
    lengths, more = [70, 130, 100], dict(window=40, sinks=2)
    off = offsets_of(lengths).cuda()
    c, dy = cuda(a), dy.cuda()
    y, lse = tcu.window_attention(**c, offsets=off, lse=True, **more)
    g = tcu.window_attention_grad(dy, **c, y=y, lse=lse, offsets=off, **more)
    i = torch.arange(300)
    begin = torch.repeat_interleave(torch.tensor([0, 70, 200]), torch.tensor(lengths))
    sees = ref.visible((i - begin)[:, None], (i - begin)[None], 40, 2) & (begin[:, None] == begin)
    sees = sees.cuda()
    for name in ("v", "k", "q"):
        d = {n: t.clone() for n, t in c.items()}
        d[name][where] = bad
        y2, lse2 = tcu.window_attention(**d, offsets=off, lse=True, **more)
        touched = sees[:, where] if name != "q" else i.cuda() == where
        assert torch.equal(y2[~touched], y[~touched]), name
        if name == "v":
            assert not y2[touched].isfinite().all(-1).any()
        g2 = tcu.window_attention_grad(dy, **d, y=y2, lse=lse2, offsets=off, **more)
        assert torch.equal(g2.q[~touched], g.q[~touched]), name
        # keys that a touched row sees
        reached = (sees & touched[:, None]).any(0)
        assert torch.equal(g2.k[~reached], g.k[~reached]), name
        assert torch.equal(g2.v[~reached], g.v[~reached]), name
    e = dy.clone()
    e[where] = bad
    g2 = tcu.window_attention_grad(e, **c, y=y, lse=lse, offsets=off, **more)
    rest = i.cuda() != where
    assert torch.equal(g2.q[rest], g.q[rest])
    assert torch.equal(g2.k[~sees[where]], g.k[~sees[where]])
    assert torch.equal(g2.v[~sees[where]], g.v[~sees[where]])
    assert not g2.v[sees[where]].isfinite().all(-1).any()


@gpu
@pytest.mark.parametrize("dtype", HALF)
def test_rows_out_of_sight_may_be_anything(tcu, dtype):
    """Keys and values that no row of a tile sees are not read; keys that a
    row does not see do not reach it, whatever they are."""
    a, _ = inputs(dtype, (1, 700), 2, 1, 64)
    c = cuda(a)
    y = tcu.window_attention(**c, window=100)
    c["k"][:, :300], c["v"][:, :200] = float("nan"), float("nan")
    y2 = tcu.window_attention(**c, window=100)
    assert torch.equal(y2[:, 400:], y[:, 400:])
    c["k"][:, 650:] = float("inf")
    assert torch.equal(tcu.window_attention(**c, window=100)[:, 400:650], y[:, 400:650])


@gpu
def test_nothing_to_do(tcu):
    for dtype in HALF:
        q = torch.zeros(2, 0, 4, 64, dtype=dtype, device="cuda")
        y, lse = tcu.window_attention(q, q, q, window=4, lse=True)
        assert y.shape == q.shape and lse.shape == (2, 0, 4)
        assert tcu.window_attention_grad(q, q, q, q, y, lse, window=4).k.shape == q.shape
        off = torch.zeros(4, dtype=torch.int32, device="cuda")
        p = torch.full((5, 4, 64), float("nan"), dtype=dtype, device="cuda")
        out = torch.ones_like(p)
        _, lse = tcu.window_attention(p, p, p, window=4, offsets=off, lse=True, out=out)
        assert (out == 1).all()
        for t in tcu.window_attention_grad(p, p, p, p, p, lse, window=4, offsets=off):
            assert (t == 0).all()


@gpu
@pytest.mark.parametrize("dtype", HALF)
@pytest.mark.parametrize("heads,kv,dim,window,sinks,length", [
    (4, 2, 64, 20, 3, 60), (1, 1, 128, 100, 0, 130), (6, 2, 80, 16, 5, 18), (40, 2, 128, 33, 1, 50),
    (8, 8, 8, 7, 0, 20), (4, 1, 128, 300, 10, 400), (16, 1, 96, 1, 0, 5), (3, 1, 64, 1500, 4, 700)])
def test_tokens_continue_a_prompt(tcu, dtype, heads, kv, dim, window, sinks, length):
    """A cache filled from a prompt's first rows, then a token at a time: each
    row as the whole prompt gives it."""
    u = U[dtype]
    a, _ = inputs(dtype, (2, length), heads, kv, dim)
    want, _ = ref.attention(**{n: t.double() for n, t in a.items()}, window=window, sinks=sinks)
    c = cuda(a)
    more = dict(window=window, sinks=sinks)
    slots = torch.tensor([4, 1], dtype=torch.int32, device="cuda")
    start = length - min(length, 25)
    # memory that no row has entered is no number, and is not read
    ck, cv = torch.full((2, 5, sinks + window, kv, dim), float("nan"), dtype=dtype, device="cuda")
    tcu.window_cache(c["k"][:, :start], c["v"][:, :start], ck, cv, slots=slots, **more)
    for t in range(start, length):
        place = torch.full((2,), t, dtype=torch.int32, device="cuda")
        y = tcu.window_attention_step(c["q"][:, t], c["k"][:, t], c["v"][:, t], ck, cv, place,
                                      slots=slots, **more)
        close(y, want[:, t], t, u + 2e-5)
    full_k, full_v = torch.full((2, 5, sinks + window, kv, dim), float("nan"), dtype=dtype, device="cuda")
    tcu.window_cache(c["k"], c["v"], full_k, full_v, slots=slots, **more)
    for got, filled in ((ck, full_k), (cv, full_v)):
        assert torch.equal(got.view(torch.int16), filled.view(torch.int16))
        assert got[[0, 2, 3]].isnan().all()


@gpu
@pytest.mark.parametrize("dtype", HALF)
def test_caches_of_packed_prompts(tcu, dtype):
    lengths, window, sinks = [3, 0, 40, 1, 25], 11, 4
    a, _ = inputs(dtype, (sum(lengths) + 6,), 2, 2, 16)
    c, off = cuda(a), offsets_of(lengths)
    slots = torch.tensor([2, 6, 0, 9, -1], dtype=torch.int32).cuda()
    ck, cv = torch.zeros(2, 7, sinks + window, 2, 16, dtype=dtype, device="cuda")
    want_k, want_v = ck.cpu(), cv.cpu()
    for s, slot in ((0, 2), (1, 6), (2, 0)):  # the others are outside
        lo, n = off[s].item(), lengths[s]
        for p in range(n):
            if p < sinks or n - p <= window:
                row = p if p < sinks else sinks + (p - sinks) % window
                want_k[slot, row], want_v[slot, row] = a["k"][lo + p], a["v"][lo + p]
    tcu.window_cache(c["k"], c["v"], ck, cv, window=window, sinks=sinks, offsets=off.cuda(), slots=slots)
    assert torch.equal(ck.cpu(), want_k) and torch.equal(cv.cpu(), want_v)


@gpu
@pytest.mark.parametrize("dtype", HALF)
def test_tokens_outside(tcu, dtype):
    """Slots outside the caches and positions below zero: rows of zeros, caches
    as they were; other rows at the largest position."""
    gen = torch.Generator().manual_seed(0)
    q, k = randn(gen, 4, 4, 64, dtype=dtype).cuda(), randn(gen, 4, 2, 64, dtype=dtype).cuda()
    cache = randn(gen, 2, 3, 9, 2, 64, dtype=dtype).cuda()
    kept = cache.clone()
    slots = torch.tensor([-1, 3, 1, 2], dtype=torch.int32, device="cuda")
    place = torch.tensor([5, 5, -1, 2 ** 31 - 1], dtype=torch.int32, device="cuda")
    y = tcu.window_attention_step(q, k, k, *cache.unbind(0), place, window=7, sinks=2, slots=slots)
    assert (y[:3] == 0).all() and torch.equal(cache[:, :2], kept[:, :2])
    row = 2 + (2 ** 31 - 3) % 7
    kept[:, 2, row] = k[3]
    assert torch.equal(cache, kept)
    ks, vs = (t[2].double().cpu().repeat_interleave(2, 1) for t in cache.unbind(0))
    p = torch.softmax(torch.einsum("hd,nhd->hn", q[3].double().cpu(), ks) / 8, -1)
    close(y[3], torch.einsum("hn,nhd->hd", p, vs), inner=U[dtype] + 2e-5)


@gpu
@pytest.mark.parametrize("dtype", HALF)
def test_large_batches_of_tokens(tcu, dtype):
    """Many entries: no clusters; one entry of a long window: clusters of 8."""
    for batch, window, kv in ((700, 40, 2), (1, 5000, 1), (20, 900, 4)):
        gen = torch.Generator().manual_seed(0)
        q = randn(gen, batch, 4 * kv, 64, dtype=dtype).cuda()
        k, v = randn(gen, 2, batch, kv, 64, dtype=dtype).cuda()
        cache = randn(gen, 2, batch, window + 2, kv, 64, dtype=dtype).cuda()
        place = torch.randint(0, 3 * window, (batch,), generator=gen, dtype=torch.int32)
        y = tcu.window_attention_step(q, k, v, *cache.unbind(0), place.cuda(), window=window, sinks=2)
        ks, vs = (t.double() for t in cache.unbind(0))  # the new rows are in it
        score = torch.einsum("bkgd,bnkd->bkgn", q.double().unflatten(1, (kv, 4)), ks) / 8
        held = torch.arange(window + 2)[None] <= place[:, None]
        score = score.masked_fill(~held.cuda()[:, None, None], float("-inf"))
        want = torch.einsum("bkgn,bnkd->bkgd", torch.softmax(score, -1), vs).flatten(1, 2)
        close(y, want.cpu(), (batch, window), U[dtype] + 2e-5)


@gpu
def test_autograd(tcu):
    """Through autograd, gradients in any layout; inputs broadcast over rows."""
    a, dy = inputs(torch.bfloat16, (2, 140), 4, 2, 64)
    c, dy = cuda(a), dy.cuda()
    more = dict(window=50, sinks=2)
    leaves = {n: t.clone().requires_grad_() for n, t in c.items()}
    y = tcu.window_attention(**leaves, **more)
    y.backward(dy.transpose(1, 2).contiguous().transpose(1, 2))
    plain, lse = tcu.window_attention(**c, **more, lse=True)
    g = tcu.window_attention_grad(dy, **c, y=plain, lse=lse, **more)
    for n in leaves:
        assert torch.equal(leaves[n].grad, getattr(g, n)), n
    tcu.window_attention(**leaves, **more).sum().backward()  # dy of one value, expanded


@gpu
def test_differences(tcu):
    """Along a direction, by central differences of the output in 16 bits: its
    roundings, u |dy||y| sqrt(values), over the step."""
    a, dy = inputs(torch.float16, (1, 200), 2, 1, 64)
    c, dy = cuda(a), dy.cuda()
    more = dict(window=70, sinks=3)
    y, lse = tcu.window_attention(**c, **more, lse=True)
    g = tcu.window_attention_grad(dy, **c, y=y, lse=lse, **more)
    gen = torch.Generator().manual_seed(4)
    h = 0.125  # steps of fp16 values of 2^-3 are all but exact
    for n in c:
        way = (torch.randint(0, 2, c[n].shape, generator=gen) * 2 - 1).half().cuda() * h
        loss = lambda t: (tcu.window_attention(**dict(c, **{n: t}), **more).double()  # noqa: E731
                          * dy.double()).sum().item()
        up, down = c[n] + way, c[n] - way
        slope = loss(up) - loss(down)
        want = (getattr(g, n).double() * (up.double() - down.double())).sum().item()
        noise = 2 ** -11 * (dy.double() * y.double()).norm().item() * 2
        # h^2 / 6 of the third derivative, of the order of the slope's terms
        terms = (getattr(g, n).double() * 2 * h).norm().item()
        assert abs(slope - want) <= 4 * noise + 0.05 * max(abs(want), terms), n


@gpu
def test_graphs_and_streams(tcu):
    a, dy = inputs(torch.bfloat16, (300,), 4, 2, 64)
    c, dy, off = cuda(a), dy.cuda(), offsets_of([100, 0, 200]).cuda()
    more = dict(window=50, sinks=2)
    y, lse = tcu.window_attention(**c, offsets=off, lse=True, **more)
    want = (y, lse, *tcu.window_attention_grad(dy, **c, y=y, lse=lse, offsets=off, **more))
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    got = tcu.window_attention(**c, offsets=off, stream=side, **more)
    torch.cuda.current_stream().wait_stream(side)
    assert torch.equal(got, y)
    cache = torch.zeros(2, 3, 52, 2, 64, dtype=torch.bfloat16, device="cuda")
    place = torch.tensor([100, 0, 200], dtype=torch.int32, device="cuda")
    token = [c[n][:3].clone() for n in ("q", "k", "v")]

    def serve(to):
        tcu.window_cache(c["k"], c["v"], *to.unbind(0), offsets=off, **more)
        return tcu.window_attention_step(*token, *to.unbind(0), place, **more)

    expect = cache.clone()
    first = serve(expect)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        y, lse = tcu.window_attention(**c, offsets=off, lse=True, **more)
        g = tcu.window_attention_grad(dy, **c, y=y, lse=lse, offsets=off, **more)
        z = serve(cache)
    for _ in range(2):
        for t in (y, lse, *g, z, cache):
            t.fill_(3)
        cache.zero_()
        graph.replay()
        torch.cuda.synchronize()
        for x, w in zip((y, lse, *g, z, cache), (*want, first, expect)):
            assert torch.equal(x, w)


# ------------------------------------------------------------ without a GPU
@pytest.mark.parametrize("packed", [False, True])
def test_reference_against_differences(packed):
    gen = torch.Generator().manual_seed(0)
    off = offsets_of([4, 0, 2]) if packed else None
    lead = (6,) if packed else (2, 5)
    q, k, v = (torch.randn(*lead, h, 3, generator=gen, dtype=torch.float64).requires_grad_()
               for h in (2, 1, 1))
    assert torch.autograd.gradcheck(lambda *a: ref.attention(*a, 2, 1, offsets=off), (q, k, v))


def test_reference_by_hand():
    """Equal scores: means of the visible values."""
    z, v = torch.zeros(1, 5, 1, 1).double(), torch.arange(5.0).double().reshape(1, 5, 1, 1)
    y, lse = ref.attention(z, z, v, 2, 1)
    want = torch.tensor([0, 0.5, 1, 5 / 3, 7 / 3], dtype=torch.float64)
    assert torch.allclose(y.flatten(), want)
    assert torch.allclose(lse.flatten().exp(), torch.tensor([1.0, 2, 3, 3, 3], dtype=torch.float64))


def args(attn, **change):
    fake = 0x10000  # never dereferenced: every call here is refused
    r = attn._Rows(fake, 5 * 64, 64)
    v = dict(type=1, sequences=2, heads=4, kv_heads=2, dim=16, window=3, sinks=1, scale=0.25, rows=5,
             lse=fake, workspace=fake, workspace_bytes=1 << 30,
             **{k: r for k in ("q", "k", "v", "y", "dy", "dq", "dk", "dv")})
    v.update(change)
    return attn._AttentionArgs(**v)


INVALID, UNSUPPORTED = 1, 2


@pytest.mark.parametrize("call,change,status", [
    ("attention", dict(type=3), INVALID), ("attention", dict(type=0), UNSUPPORTED),
    ("attention", dict(dim=12), UNSUPPORTED), ("attention", dict(dim=136), UNSUPPORTED),
    ("attention", dict(dim=0), INVALID), ("attention", dict(heads=3), INVALID),
    ("attention", dict(kv_heads=0), INVALID), ("attention", dict(window=0), INVALID),
    ("attention", dict(sinks=-1), INVALID), ("attention", dict(scale=0.0), INVALID),
    ("attention", dict(scale=float("nan")), INVALID), ("attention", dict(scale=float("inf")), INVALID),
    ("attention", dict(rows=2 ** 31), UNSUPPORTED), ("attention", dict(lse=0x10002), INVALID),
    ("attention", dict(offsets=0x10001), INVALID), ("attention", dict(sequences=-1), INVALID),
    ("attention_grad", dict(lse=None), INVALID), ("attention_grad", dict(workspace_bytes=8), INVALID),
    ("attention_grad", dict(workspace=None), INVALID),
    ("attention_step", dict(), INVALID),  # five rows
    ("attention_step", dict(rows=1, num_slots=1), INVALID),
    ("attention_step", dict(rows=1, num_slots=2, positions=0x10000), INVALID),  # no caches
    ("attention_step", dict(rows=1, num_slots=2, cache_k=0x90000, cache_v=0xa0000), INVALID),
    ("attention_step", dict(rows=1, num_slots=2, cache_k=0x90000, cache_v=0x90100,
                            positions=0x10000), INVALID),  # over each other
    ("attention_step", dict(rows=1, num_slots=2, cache_k=0x10000, cache_v=0xa0000,
                            positions=0xf0000), INVALID),  # over the rows
    ("attention_step", dict(rows=1, num_slots=2, cache_k=0x90008, cache_v=0xa0000,
                            positions=0xf0000), INVALID),
    ("cache", dict(num_slots=1), INVALID), ("cache", dict(num_slots=2), INVALID),
    ("cache", dict(num_slots=2, cache_k=0x10000, cache_v=0xa0000), INVALID)])
def test_refusals(tcu, call, change, status):
    from paper_1908_06649_gb300 import attention as attn
    assert getattr(attn._lib(), "tcu_window_" + call)(args(attn, **change), None) == status


def test_refused_rows(tcu):
    from paper_1908_06649_gb300 import attention as attn
    L, R = attn._lib(), attn._Rows
    for bad, status in ((R(0x10000, 2 ** 33, 2 ** 31), UNSUPPORTED), (R(0x10008, 320, 64), INVALID),
                        (R(0x10000, 320, 60), INVALID), (R(0x10000, 320, 24), INVALID),
                        (R(0x10000, 324, 64), INVALID), (R(0x10000, 320, -64), INVALID),
                        (R(0x10000, 0, 64), INVALID), (R(0, 320, 64), INVALID)):
        for k in ("q", "k", "v", "y"):
            assert L.tcu_window_attention(args(attn, **{k: bad}), None) == status, (k, bad)
        for k in ("dy", "dq", "dk", "dv"):
            assert L.tcu_window_attention_grad(args(attn, **{k: bad}), None) == status, (k, bad)
    assert L.tcu_window_attention(None, None) == INVALID
    assert L.tcu_window_attention_grad_workspace(args(attn)) > 0
    assert L.tcu_window_attention_grad_workspace(args(attn, dim=9)) == -1


@gpu
def test_refusals_of_tensors(tcu):
    q = torch.zeros(2, 5, 4, 16, dtype=torch.bfloat16, device="cuda")
    k = q[:, :, :2].contiguous()
    ok = dict(q=q, k=k, v=k, window=3)
    y, lse = tcu.window_attention(**ok, lse=True)
    wide = torch.zeros(2, 5, 4, 20, dtype=torch.bfloat16, device="cuda")
    for bad in (dict(q=q.cpu()), dict(q=q.float()), dict(k=k.half()), dict(k=k[:, :4]), dict(v=q),
                dict(k=q[:, :, :3], v=q[:, :, :3]), dict(window=0), dict(sinks=-1), dict(scale=0.0),
                dict(scale=float("inf")), dict(q=q[0]), dict(out=q), dict(q=wide[..., :16]),
                dict(q=q[:1].expand(2, 5, 4, 16)), dict(q=q[..., :12], k=k[..., :12], v=k[..., :12]),
                dict(q=q.transpose(1, 2)), dict(offsets=torch.zeros(3, device="cuda"))):
        with pytest.raises((ValueError, TypeError)):
            tcu.window_attention(**{**ok, **bad})
    with pytest.raises(ValueError):
        tcu.window_attention(q.clone().requires_grad_(), k, k, window=3, lse=True)
    with pytest.raises(ValueError):
        tcu.window_attention_grad(q, **ok, y=y, lse=lse[:, :4])
    cache = torch.zeros(2, 2, 3, 2, 16, dtype=torch.bfloat16, device="cuda")
    ck, cv = cache.unbind(0)
    place = torch.zeros(2, dtype=torch.int32, device="cuda")
    ok = dict(q=q[:, 0], k=k[:, 0], v=k[:, 0], cache_k=ck, cache_v=cv, positions=place, window=3)
    tcu.window_attention_step(**ok)
    for bad in (dict(cache_k=ck[:1]), dict(cache_v=cv.half()), dict(window=4), dict(positions=None),
                dict(positions=place.long()), dict(slots=place[:1]), dict(cache_v=ck),
                dict(out=q[:, 0]), dict(k=ck[:, 0]), dict(cache_k=ck.clone().requires_grad_()),
                dict(q=q), dict(cache_k=ck.transpose(1, 2))):
        with pytest.raises((ValueError, TypeError, tcu.TcuDftError)):
            tcu.window_attention_step(**{**ok, **bad})
    with pytest.raises((ValueError, tcu.TcuDftError)):
        tcu.window_cache(ck, ck, ck, cv, window=3)
    with pytest.raises(ValueError):
        tcu.window_cache(k, k.clone().requires_grad_(), ck, cv, window=3)
    from torch.autograd import forward_ad
    with forward_ad.dual_level():
        dual = forward_ad.make_dual(k, torch.ones_like(k))
        for call in (lambda: tcu.window_attention(q, dual, k, window=3),
                     lambda: tcu.window_attention_grad(q, q, k, dual, y, lse, window=3),
                     lambda: tcu.window_attention_step(**{**ok, "v": dual[:, 0]}),
                     lambda: tcu.window_cache(dual, k, ck, cv, window=3)):
            with pytest.raises(ValueError, match="forward-mode"):
                call()
    before = ck._version
    tcu.window_attention_step(**ok)
    assert ck._version > before


@gpu
def test_beyond_32_bits_of_elements(tcu):
    """2.2e9 values of q: the last rows are what a call on the last rows alone
    gives; so are their gradients, but for rows whose later readers are cut."""
    rows, heads, window, keep = 270000, 64, 100, 1000
    gen = torch.Generator(device="cuda").manual_seed(0)
    q = torch.empty(1, rows, heads, 128, dtype=torch.bfloat16, device="cuda").normal_(generator=gen)
    k, v = (torch.empty(1, rows, 1, 128, dtype=torch.bfloat16, device="cuda").normal_(generator=gen)
            for _ in range(2))
    y, lse = tcu.window_attention(q, k, v, window=window, lse=True)
    e = [t[:, rows - keep:].clone() for t in (q, k, v)]
    z, s = tcu.window_attention(*e, window=window, lse=True)
    u = U[torch.bfloat16]
    close(y[:, window - keep:], z[:, window:].double().cpu(), inner=2 * u + 2e-5)
    close(lse[:, window - keep:], s[:, window:].double().cpu())
    g = tcu.window_attention_grad(q, q, k, v, y, lse, window=window)
    w = tcu.window_attention_grad(e[0], *e, z, s, window=window)
    close(g.q[:, window - keep:], w.q[:, window:].double().cpu(), inner=4 * u + 2e-5)
    close(g.v[:, window - keep:], w.v[:, window:].double().cpu(), inner=4 * u + 2e-5)
    # a cache beyond as many
    del y, lse, g, q
    cache = torch.empty(2, 2200, 8000, 1, 128, dtype=torch.bfloat16, device="cuda")
    cache[:, 2199].normal_(generator=gen)
    slot = torch.tensor([2199], dtype=torch.int32, device="cuda")
    place = torch.tensor([9000], dtype=torch.int32, device="cuda")
    token = [t[:, -1] for t in e]
    far = tcu.window_attention_step(*token, *cache.unbind(0), place, window=8000, slots=slot)
    near = cache[:, 2199:].clone()
    got = tcu.window_attention_step(*token, *near.unbind(0), place, window=8000)
    assert torch.equal(far, got)
