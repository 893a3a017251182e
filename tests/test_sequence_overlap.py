"""Outputs that share memory with inputs, or with themselves, are refused;
those that lie between an input's elements are not."""
import itertools
import random

import pytest
import torch

W = 4


@pytest.fixture(scope="module")
def seq():
    from paper_1908_06649_gb300 import _build
    _build.build()
    from paper_1908_06649_gb300 import sequence
    return sequence


def touched(t, base):
    """Byte offsets of every element's bytes, with repeats."""
    size, first = t.element_size(), t.data_ptr() - base
    return [first + size * sum(i * s for i, s in zip(ix, t.stride())) + k
            for ix in itertools.product(*map(range, t.shape)) for k in range(size)]


def test_overlap_is_exact(seq):
    """Random layouts, element sizes mixed, against every byte they touch."""
    rng = random.Random(5)
    buf = torch.zeros(200, dtype=torch.int16)

    def view():
        b = rng.choice([buf, buf.view(torch.int32)])
        while True:
            shape = [rng.randint(1, 4) for _ in range(rng.randint(1, 3))]
            strides = [rng.choice([0, 1, 2, 3, 5, 6, 8, 12, 16, 24]) for _ in shape]
            if rng.random() < 0.7:
                strides[-1] = 1
            last = sum((n - 1) * s for n, s in zip(shape, strides))
            if last < b.numel():
                return torch.as_strided(b, shape, strides, rng.randrange(b.numel() - last))

    seen = [0, 0]
    for _ in range(4000):
        one, two = view(), view()
        a, b = touched(one, buf.data_ptr()), touched(two, buf.data_ptr())
        want, itself = bool(set(a) & set(b)), len(set(a)) < len(a)
        assert seq._overlap(seq._memory(one), seq._memory(two)) == want, (one.stride(), two.stride())
        assert seq._overlaps_itself(seq._memory(one)) == itself, (one.shape, one.stride())
        seen[0] += want
        seen[1] += itself
    assert min(seen) > 200


def test_batch_and_rows_swapped(seq):
    """out[0] is the memory of x[1]."""
    buf = torch.zeros(5, 4, 8)
    with pytest.raises(ValueError):
        seq._apart(buf[:, 1:].transpose(0, 1), (buf[:, :3].transpose(0, 1),))
    # columns of the same rows, and batch entries of their own, are apart
    seq._apart(buf[..., 4:].transpose(0, 1), (buf[..., :4].transpose(0, 1),))
    seq._apart(buf[:, 2:].transpose(0, 1), (buf[:, :2].transpose(0, 1),))
    seq._apart(buf[:, 2:], (buf[:, :2],))
    seq._apart(buf[::2], (buf[1::2],))


@pytest.mark.gpu
def test_outputs_of_prompts(seq):
    b, t, c, n = 2, 20, 16, 8
    u, dt, gate = (torch.randn(b, t, c, device="cuda") for _ in range(3))
    A, skip = -torch.rand(c, n, device="cuda"), torch.randn(c, device="cuda")
    room = torch.randn(b * t * c + 4096, device="cuda")
    out = room[:b * t * c].view(b, t, c)
    B, C = torch.randn(b, t, 1, n, device="cuda"), torch.randn(b, t, 1, n, device="cuda")
    state = torch.randn(b, c, n, device="cuda")
    ok = dict(u=u, dt=dt, A=A, B=B, C=C, skip=skip, gate=gate, dt_bias=skip.clone(), state=state)

    def scan(to, **change):
        v = dict(ok, **change)
        return seq.state_scan(*[v.pop(k) for k in "u dt A B C".split()], out=to, **v)[0]

    want = scan(None)
    assert torch.equal(scan(out), want)
    for k, v in ok.items():  # each argument in turn at the end of the output's memory
        room.copy_(torch.randn_like(room))
        moved = room[out.numel() - 4:][:v.numel()].view(v.shape)
        with pytest.raises(ValueError):
            scan(out, **{k: moved})
        scan(out, **{k: room[out.numel():][:v.numel()].view(v.shape)})
    # an output over itself
    for to in (u.new_empty(1, t, c).expand(b, t, c), u.new_empty(b, 1, c).expand(b, t, c),
               torch.as_strided(room, (b, t, c), (t * c, c - 1, 1))):
        with pytest.raises(ValueError):
            scan(to)
        with pytest.raises(ValueError):
            seq.short_conv(u, torch.randn(c, W, device="cuda"), out=to)
    # the columns beside B and C in the projection that holds them
    wide = torch.randn(b, t, c + 2 * n, device="cuda")
    beside = dict(B=wide[..., c:c + n].unsqueeze(-2), C=wide[..., c + n:].unsqueeze(-2))
    want = scan(None, **beside)
    assert torch.equal(scan(wide[..., :c], **beside), want)
    with pytest.raises(ValueError):
        scan(wide[..., 1:c + 1], **beside)
    x = torch.randn(b, t, c, device="cuda")
    weight = room[out.numel() - 4:][:c * W].view(c, W)
    with pytest.raises(ValueError):
        seq.short_conv(x, weight, out=out)
    history = torch.randn(b * t * c, device="cuda")
    with pytest.raises(ValueError):
        seq.short_conv(x, A[:, :W].contiguous(), state=history[:b * (W - 1) * c].view(b, W - 1, c),
                       out=history.view(b, t, c))


@pytest.mark.gpu
def test_outputs_of_tokens(seq):
    """One row may be overwritten by its own result; nothing else may."""
    b, c, n = 5, 16, 8
    u, dt, gate = (torch.randn(b, c, device="cuda") for _ in range(3))
    A = -torch.rand(c, n, device="cuda")
    B, C = torch.randn(b, n, device="cuda"), torch.randn(b, n, device="cuda")
    first = torch.randn(b, c, n, device="cuda")

    def scan(to, state=None, **change):
        v = dict(dict(u=u, dt=dt, B=B, C=C), **change)
        return seq.state_scan_step(v["u"], v["dt"], A, v["B"], v["C"],
                                   first.clone() if state is None else state, gate=gate, out=to)

    want = scan(None)
    for k in ("u", "dt"):
        mine = dict(u=u, dt=dt)[k].clone()
        assert torch.equal(scan(mine, **{k: mine}), want)
    wide = torch.randn(b + 1, 2 * c, device="cuda")
    wide[:b, :c] = u
    assert torch.equal(scan(wide[:b, c:], u=wide[:b, :c]), want)
    for to in (wide[1:, :c], wide[:b, 1:c + 1]):
        with pytest.raises(ValueError):
            scan(to, u=wide[:b, :c])
    cache = first.clone()
    room = torch.randn(b, 2 * n, device="cuda")
    for to, change in ((cache.view(-1)[:b * c].view(b, c), dict(state=cache)),
                       (room.view(-1)[:b * c].view(b, c), dict(B=room[:, :n])),
                       (u.new_empty(1, c).expand(b, c), {})):
        with pytest.raises(ValueError):
            scan(to, **change)
    assert torch.equal(cache, first)
    w, past = torch.randn(c, W, device="cuda"), torch.randn(b, W - 1, c, device="cuda")
    want = seq.short_conv_step(u, past.clone(), w)
    x = u.clone()
    assert torch.equal(seq.short_conv_step(x, past.clone(), w, out=x), want)
    for to in (past.view(-1)[:b * c].view(b, c), wide[1:, :c]):
        with pytest.raises(ValueError):
            seq.short_conv_step(wide[:b, :c], past, w, out=to)


@pytest.mark.gpu
def test_caches_over_other_arguments(seq):
    """A cache that a token call advances shares memory with no other argument;
    it may lie between the rows of one."""
    from paper_1908_06649_gb300 import TcuDftError
    b, c, n = 3, 16, 8
    size = b * c * n
    arena = torch.randn(8 * size, device="cuda")
    ok = dict(u=torch.randn(b, c, device="cuda"), dt=torch.randn(b, c, device="cuda"),
              A=-torch.rand(c, n, device="cuda"), B=torch.randn(b, n, device="cuda"),
              C=torch.randn(b, n, device="cuda"), gate=torch.randn(b, c, device="cuda"),
              skip=torch.randn(c, device="cuda"), dt_bias=torch.randn(c, device="cuda"),
              slots=torch.arange(b, device="cuda").int())

    def scan(cache, **change):
        v = dict(ok, **change)
        return seq.state_scan_step(*[v.pop(k) for k in "u dt A B C".split()], cache, **v)

    def at(first, like):
        return arena[first:first + like.numel()].view(like.shape)

    first = arena[size:2 * size].view(b, c, n)
    start = first.clone()
    want = scan(start.clone())
    for k, v in ok.items():
        for where in (size - v.numel() + 1, size + 8, 2 * size - 1):
            t = at(where, v) if k != "slots" else arena.view(torch.int32)[where:where + b]
            with pytest.raises(TcuDftError):
                scan(first, **{k: t})
        t = at(2 * size, v) if k != "slots" else arena.view(torch.int32)[2 * size:2 * size + b]
        t.copy_(v)
        cache = arena[size:2 * size].view(b, c, n).copy_(start)
        assert torch.equal(scan(cache, **{k: t}), want), k
    # between the first and the second row of u
    apart = arena[:b * 2 * size].view(b, 2 * size)[:, :c].copy_(ok["u"])
    cache = arena[c:c + size].view(b, c, n).copy_(start)
    assert torch.equal(scan(cache, u=apart), want)
    with pytest.raises(TcuDftError):
        scan(arena[2 * size - size + 1:2 * size + 1].view(b, c, n), u=apart)
    x, w = torch.randn(b, c, device="cuda"), torch.randn(c, W, device="cuda")
    past = arena[:b * (W - 1) * c].view(b, W - 1, c)
    for x1, w1 in ((at(past.numel() - 1, x), w), (x, at(past.numel() - 1, w))):
        with pytest.raises(TcuDftError):
            seq.short_conv_step(x1, past, w1)
