"""Gradients of window attention where inputs span the range of their type:
rows, sequences and batch entries whose dy differ by up to 2^18, values near
the type's largest, weights below fp16's normal range.

Each part is held to its own size, with the tolerances of
test_window_attention.py (3 u before the last rounding): what a row or a key
does not see has no say in its gradients' precision, and rounding is relative
to what is rounded, whatever its size."""
import pytest
import torch

import mixing_reference as ref
from mixing_reference import U, close, cuda, offsets_of, randn

gpu = pytest.mark.gpu
HALF = [torch.bfloat16, torch.float16]


@pytest.fixture(scope="module")
def tcu():
    from paper_1908_06649_gb300 import _build
    _build.build()
    import paper_1908_06649_gb300 as p
    p.lib()
    return p


def inputs(dtype, lead, heads, kv, dim, seed=0):
    gen = torch.Generator().manual_seed(seed)
    r = lambda h: randn(gen, *lead, h, dim, dtype=dtype)  # noqa: E731
    return dict(q=r(heads), k=r(kv), v=r(kv)), r(heads)


def check_parts(tcu, a, dy, window, sinks, parts, offsets=None):
    """parts: for q, k and v a list of what is compared on its own."""
    u = U[dy.dtype]
    d = {n: t.double().requires_grad_() for n, t in a.items()}
    want, _ = ref.attention(**d, window=window, sinks=sinks, offsets=offsets)
    grads = torch.autograd.grad(want, list(d.values()), dy.double())
    with torch.no_grad():
        terms = ref.attention_terms(**d, dy=dy.double(), window=window, sinks=sinks, offsets=offsets)
    more = dict(window=window, sinks=sinks, offsets=None if offsets is None else offsets.cuda())
    c = cuda(a)
    y, lse = tcu.window_attention(**c, **more, lse=True)
    g = tcu.window_attention_grad(dy.cuda(), **c, y=y, lse=lse, **more)
    for n, got, exact, sizes in zip(g._fields, g, grads, terms):
        for at in parts[n]:
            # what the type's range does not hold is not compared (1 %: 4 u in fp16 is 0.2 %)
            fits = exact[at].abs() < 0.99 * torch.finfo(dy.dtype).max
            close(got.cpu()[at][fits], exact[at][fits], ("d" + n, at), 3 * u + 2e-5, sizes[at][fits])
    for x, z in zip(g, tcu.window_attention_grad(dy.cuda(), **c, y=y, lse=lse, **more)):
        assert torch.equal(x, z)


@gpu
@pytest.mark.parametrize("dtype", HALF)
@pytest.mark.parametrize("high,low", [(0, 0), (8, -4), (10, -4), (12, -6)])
@pytest.mark.parametrize("dim,window,sinks", [(64, 600, 0), (128, 90, 3)])
def test_batch_entries_of_other_sizes(tcu, dtype, high, low, dim, window, sinks):
    a, dy = inputs(dtype, (2, 600), 2, 1, dim)
    dy[0] *= 2.0 ** high
    dy[1] *= 2.0 ** low
    both = [(0,), (1,)]
    check_parts(tcu, a, dy, window, sinks, dict(q=both, k=both, v=both))


@gpu
@pytest.mark.parametrize("dtype", HALF)
@pytest.mark.parametrize("window,sinks", [(1000, 0), (30, 2)])
def test_packed_sequences_of_other_sizes(tcu, dtype, window, sinks):
    """Sequences that share tiles."""
    lengths, sizes = [200, 37, 300, 63, 20, 80], [12, -6, 10, -4, -6, 12]
    off = offsets_of(lengths)
    a, dy = inputs(dtype, (sum(lengths),), 4, 2, 80)
    parts = [(slice(off[s].item(), off[s + 1].item()),) for s in range(len(lengths))]
    for at, e in zip(parts, sizes):
        dy[at] *= 2.0 ** e
    check_parts(tcu, a, dy, window, sinks, dict(q=parts, k=parts, v=parts), off)


@gpu
@pytest.mark.parametrize("dtype", HALF)
@pytest.mark.parametrize("row", [5, 100, 700])
def test_one_row_of_another_size(tcu, dtype, row):
    """A row's dy 2^17 times the others': other rows' dq, and dk and dv of the
    keys that it does not see, lose nothing."""
    a, dy = inputs(dtype, (1, 1024), 2, 1, 64)
    dy *= 0.125
    dy[:, row] *= 2.0 ** 17
    rest, behind = [(0, slice(0, row)), (0, slice(row + 1, None))], [(0, slice(row + 1, None))]
    check_parts(tcu, a, dy, 1024, 0, dict(q=rest, k=behind, v=behind))


@gpu
@pytest.mark.parametrize("dtype", HALF)
def test_heads_of_other_sizes(tcu, dtype):
    """Key heads apart; query heads that share one add up to its dk and dv."""
    a, dy = inputs(dtype, (1, 300), 4, 2, 64)
    dy[:, :, :2] *= 2.0 ** 12
    dy[:, :, 2:] *= 2.0 ** -6
    parts = [(0, slice(None), h) for h in range(2)]
    check_parts(tcu, a, dy, 100, 2, dict(q=[(0, slice(None), h) for h in range(4)], k=parts, v=parts))


@gpu
@pytest.mark.parametrize("dtype", HALF)
def test_large_values(tcu, dtype):
    """dp of 8e5, beyond fp16's largest, where dy is at most one: each row's dy
    along its own value, two values to a row.  238 values of dk are beyond it
    too."""
    a, dy = inputs(dtype, (1, 200), 1, 1, 128)
    a["v"] = (a["v"] * 8000).clamp(-60000, 60000)
    a["k"] *= 0.25
    dy = 0.99 * torch.sign(a["v"])
    every = [(0,)]
    check_parts(tcu, a, dy, 2, 0, dict(q=every, k=every, v=every))


@gpu
@pytest.mark.parametrize("dtype", HALF)
@pytest.mark.parametrize("length", [20000, 65536])
def test_weights_of_long_rows(tcu, dtype, length):
    """Equal scores: weights of 1 / (i + 1), at the end below fp16's normal
    range; the last eighth of rows and keys is compared.  p or ds is rounded,
    and then the result: errors of random sign, 0.58 u of a value at most in
    the root mean square (uniform within half a step) and 0.4 u of many values
    of all sizes, together 0.7 u of the norm.  delta comes from a rounded y,
    but |y| is |v| / sqrt(i + 1) here, nothing beside dp.  Value by value it is
    u of the sum of the terms' sizes."""
    dim = 64
    gen = torch.Generator().manual_seed(0)
    q, k, v, dy = (randn(gen, 1, length, 1, dim, dtype=dtype).cuda() for _ in range(4))
    none, late = torch.zeros_like(q), length - length // 8

    def grads(q, k):
        y, lse = tcu.window_attention(q, k, v, window=length, lse=True)
        g = tcu.window_attention_grad(dy, q, k, v, y, lse, window=length)
        return [t[0, late:, 0] for t in g]

    qs, ks, vs, dys = (t.double()[0, :, 0] for t in (q, k, v, dy))
    want, terms = torch.zeros(2, 3, length - late, dim, dtype=torch.float64, device="cuda").unbind(0)
    for at in range(late, length, 1024):
        i = torch.arange(at, min(at + 1024, length), device="cuda")
        p = (torch.arange(length, device="cuda") <= i[:, None]) / (i[:, None] + 1.0).double()
        y = p @ vs
        ds = p * (dys[i] @ vs.T - (dys[i] * y).sum(1, keepdim=True)) / 8
        size = ds.abs() + p * (dys[i] * y).abs().sum(1, keepdim=True) / 8
        want[0][i - late], terms[0][i - late] = ds @ ks, size @ ks.abs()
        for w, s, q_ in ((want, ds, qs), (terms, size, qs.abs())):
            w[1] += s[:, late:].T @ q_[i]
        want[2] += p[:, late:].T @ dys[i]
        terms[2] += p[:, late:].T @ dys[i].abs()
    want, terms = want.cpu(), terms.cpu()
    _, dk, dv = grads(q, none)
    close(dv, want[2], "dv", terms=terms[2])
    close(dk, want[1], "dk", terms=terms[1])
    dq, _, _ = grads(none, k)
    close(dq, want[0], "dq", terms=terms[0])


@gpu
@pytest.mark.parametrize("dtype", HALF)
@pytest.mark.parametrize("dim,window", [(64, 200), (128, 3000)])
def test_tokens_are_rounded_once(tcu, dtype, dim, window):
    """Weights go to their product in two parts, u^2 of themselves off, so that
    only the result is rounded: its errors, uniform within half a step over
    values of all sizes, are 0.4 u of the norm, and half of u holds them."""
    gen = torch.Generator().manual_seed(0)
    batch, heads, kv = 16, 8, 2
    q = randn(gen, batch, heads, dim, dtype=dtype).cuda()
    k, v = (randn(gen, batch, kv, dim, dtype=dtype).cuda() for _ in range(2))
    cache = randn(gen, 2, batch, window, kv, dim, dtype=dtype).cuda()
    place = torch.full((batch,), 2 * window, dtype=torch.int32, device="cuda")
    y = tcu.window_attention_step(q, k, v, *cache.unbind(0), place, window=window)
    ks, vs = (t.double() for t in cache.unbind(0))
    score = torch.einsum("bkgd,bnkd->bkgn", q.double().unflatten(1, (kv, -1)), ks) / dim ** 0.5
    want = torch.einsum("bkgn,bnkd->bkgd", torch.softmax(score, -1), vs).flatten(1, 2)
    err = (y.double() - want).norm() / want.norm()
    assert err <= 0.5 * U[dtype], float(err / U[dtype])


@gpu
@pytest.mark.parametrize("dtype", HALF)
@pytest.mark.parametrize("length,window,sinks", [(300, 4, 0), (300, 16, 2), (500, 60, 3), (700, 180, 0)])
def test_gradients_are_rounded_twice(tcu, dtype, length, window, sinks):
    """What is rounded before the result is ds, or p, once: two errors of random
    sign, uniform within half a step over values of all sizes, 0.4 u of the norm
    each, 0.56 u in all.  delta as it comes from the rounded y would add as much
    where a row sees few keys, but there it is formed again; where it sees
    more than 256, |y| is a fraction of |v|.  0.75 u holds a third of that again."""
    a, dy = inputs(dtype, (2, length), 4, 2, 128)
    d = {n: t.double().requires_grad_() for n, t in a.items()}
    want, _ = ref.attention(**d, window=window, sinks=sinks)
    grads = torch.autograd.grad(want, list(d.values()), dy.double())
    more, c = dict(window=window, sinks=sinks), cuda(a)
    y, lse = tcu.window_attention(**c, **more, lse=True)
    g = tcu.window_attention_grad(dy.cuda(), **c, y=y, lse=lse, **more)
    for n, got, exact in zip(g._fields, g, grads):
        off = float((got.cpu().double() - exact).norm() / exact.norm() / U[dtype])
        assert off <= 0.75, (n, off)


@gpu
@pytest.mark.parametrize("dtype", HALF)
@pytest.mark.parametrize("lengths,window,sinks", [([2600], 100, 3), ([700, 0, 1990, 50], 60, 130),
                                                  ([100, 2300], 900, 4)])
def test_first_tokens_of_long_sequences(tcu, dtype, lengths, window, sinks):
    """Keys that thousands of rows see, whose sums are formed in parts: late
    rows' dy a thousandth of early ones', sequences of other sizes."""
    a, dy = inputs(dtype, (sum(lengths),), 4, 2, 64)
    off = offsets_of(lengths)
    parts = []
    for s, n in enumerate(lengths):
        at = slice(off[s].item(), off[s + 1].item())
        dy[at] *= 2.0 ** (8 if s % 2 else -2)
        dy[at.start + n // 2:at.stop] *= 2.0 ** -10
        parts += [(slice(at.start, at.start + n // 2),), (slice(at.start + n // 2, at.stop),)] if n else []
    check_parts(tcu, a, dy, window, sinks, dict(q=parts, k=parts, v=parts), off)


@gpu
def test_captured_calls_of_other_sizes(tcu):
    """One graph, replayed for inputs of other sizes: nothing is kept from one
    replay for the next."""
    a, dy = inputs(torch.float16, (2, 300), 4, 2, 64)
    c, more = cuda(a), dict(window=60, sinks=2)
    dy = dy.cuda()
    y, lse = tcu.window_attention(**c, lse=True, **more)
    static, graph = dy.clone(), torch.cuda.CUDAGraph()
    tcu.window_attention_grad(static, **c, y=y, lse=lse, **more)
    with torch.cuda.graph(graph):
        g = tcu.window_attention_grad(static, **c, y=y, lse=lse, **more)
    for e in (12, -6, 12, 0):
        static.copy_(dy * 2.0 ** e)
        graph.replay()
        want = tcu.window_attention_grad(static, **c, y=y, lse=lse, **more)
        torch.cuda.synchronize()
        for x, w in zip(g, want):
            assert torch.equal(x, w), e
