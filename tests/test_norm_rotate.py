"""The norm of heads with the rotation by position on the GPU against its
definition in 64 bits (mixing_reference.py); and what it refuses.

Tolerances, set before the first run.  Sums over at most 256 values, a
reciprocal root and a turn in fp32 are some 20 roundings of 2^-24 each, and an
angle is off by 2^-32 turns and its sine by two steps: 2e-6 at most; the
gradient doubles it, and sums over rows and heads of random sign add 2^-24
times the root of their number.  2e-5 holds all of it."""
import ctypes

import pytest
import torch

import mixing_reference as ref
from mixing_reference import TYPES, close, cuda, offsets_of, packed_lengths, randn

gpu = pytest.mark.gpu


@pytest.fixture(scope="module")
def tcu():
    from paper_1908_06649_gb300 import _build
    _build.build()
    import paper_1908_06649_gb300 as p
    p.lib()
    return p


def inputs(dtype, lead, heads, kv, dim, turned, weights=True, positions=None, offsets=None, seed=0):
    gen = torch.Generator().manual_seed(seed)
    r = lambda *s, **k: randn(gen, *s, **k)  # noqa: E731
    a = dict(q=r(*lead, heads, dim, dtype=dtype, scale=2), k=r(*lead, kv, dim, dtype=dtype),
             rates=100.0 ** -(torch.arange(turned) / turned),
             q_weight=r(dim, shift=1, scale=0.3) if weights else None,
             k_weight=r(dim, shift=1, scale=0.3) if weights else None,
             positions=positions, offsets=offsets)
    return a, r(*lead, heads, dim, dtype=dtype), r(*lead, kv, dim, dtype=dtype)


def reference(a, eps, interleaved, dq=None, dk=None):
    place = a["positions"] if a["positions"] is not None else ref.positions_of(a["q"], a["offsets"])
    outs, grads, weights = [], [], []
    for x, w, g in ((a["q"], a["q_weight"], dq), (a["k"], a["k_weight"], dk)):
        x = x.detach().double().requires_grad_()
        w = None if w is None else w.detach().double().requires_grad_()
        y = ref.norm_rotate(x, w, a["rates"].double(), place, eps, interleaved)
        outs.append(y.detach())
        if g is not None:
            got = torch.autograd.grad(y, [x] if w is None else [x, w], g.double())
            grads.append(got[0])
            weights.append(None if w is None else got[1])
    return outs, grads, weights


def check(tcu, a, dq, dk, eps=1e-6, interleaved=False):
    outs, grads, weights = reference(a, eps, interleaved, dq, dk)
    c, more = cuda(a), dict(eps=eps, interleaved=interleaved)
    for got, want in zip(tcu.norm_rotate(**c, **more), outs):
        close(got, want)
    g = tcu.norm_rotate_grad(dq.cuda(), dk.cuda(), **c, **more)
    for got, want, name in zip(g, grads + weights, g._fields):
        if want is None:
            assert got is None
        else:
            close(got, want, name)
    for x, y in zip(g, tcu.norm_rotate_grad(dq.cuda(), dk.cuda(), **c, **more)):
        assert x is y is None or torch.equal(x, y)


SIZES = [(2, 17, 4, 2, 64, 32), (1, 5, 3, 1, 128, 64), (3, 9, 7, 7, 80, 20), (2, 3, 1, 1, 2, 1),
         (1, 33, 5, 2, 6, 2), (2, 4, 2, 1, 256, 128), (1, 7, 9, 3, 96, 24), (1, 4, 3, 2, 254, 100),
         (1, 6, 2, 2, 72, 5)]


@gpu
@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("batch,length,heads,kv,dim,turned", SIZES)
def test_dense(tcu, dtype, interleaved, batch, length, heads, kv, dim, turned):
    a, dq, dk = inputs(dtype, (batch, length), heads, kv, dim, turned, weights=length != 4)
    check(tcu, a, dq, dk, interleaved=interleaved)


@gpu
@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("kind", ["one", "empties", "singles", "mixed"])
def test_packed(tcu, dtype, kind):
    off = offsets_of(packed_lengths(77, kind))
    check(tcu, *inputs(dtype, (77,), 4, 2, 64, 16, offsets=off), eps=1e-2)


@gpu
@pytest.mark.parametrize("dtype", TYPES)
def test_tokens_at_positions(tcu, dtype):
    place = torch.tensor([0, 5, 2 ** 20 + 3, 2 ** 31 - 1, -7], dtype=torch.int32)
    check(tcu, *inputs(dtype, (5,), 4, 2, 128, 64, positions=place))
    gen = torch.Generator().manual_seed(1)
    place = torch.randint(0, 2 ** 31 - 1, (2, 9), generator=gen, dtype=torch.int32)
    a, dq, dk = inputs(dtype, (2, 9), 2, 1, 64, 32, positions=place)
    a["rates"] = randn(gen, 32, scale=30)  # rates of many turns a position, of both signs
    check(tcu, a, dq, dk)


@gpu
def test_angles_of_far_positions(tcu):
    """Heads of (1, 0) pairs come out as cosine and sine: within 2^-22 of them
    at any position."""
    n = 64
    place = torch.tensor([1, 1000, 10 ** 6, 10 ** 9, 2 ** 31 - 1, -2 ** 31], dtype=torch.int32)
    rates = 10000.0 ** (-torch.arange(n) / n)
    q = torch.cat([torch.ones(6, 1, n), torch.zeros(6, 1, n)], -1).cuda()
    y, _ = tcu.norm_rotate(q, q, rates.cuda(), positions=place.cuda(), eps=0.0)
    angle = place.double()[:, None] * rates.double()
    want = torch.cat([torch.cos(angle), torch.sin(angle)], -1) * 2 ** 0.5
    assert (y[:, 0].cpu().double() - want).abs().max() < 2 ** -21


@gpu
@pytest.mark.parametrize("dtype", TYPES)
def test_strides_and_in_place(tcu, dtype):
    """Queries and keys as slices of one projection, at odd places too, over
    batch entries in another order; results over their inputs.  Rows that are
    aligned otherwise are read in other words and their squares summed in
    another order, so it is the definition that they are compared with."""
    gen = torch.Generator().manual_seed(3)
    rates = torch.rand(8, generator=gen).cuda()
    for extra in (0, 1, 4):
        big = randn(gen, 7, 3, 160 + extra, dtype=dtype).cuda().transpose(0, 1)
        q = big[..., extra:96 + extra].unflatten(-1, (6, 16))
        k = big[..., 96 + extra:128 + extra].unflatten(-1, (2, 16))
        a = dict(q=q.cpu(), k=k.cpu(), rates=rates.cpu(), q_weight=None, k_weight=None,
                 positions=None, offsets=None)
        want, grads, _ = reference(a, 1e-6, False, a["q"], a["k"])
        got = tcu.norm_rotate(q, k, rates)
        g = tcu.norm_rotate_grad(q, k, q, k, rates)
        for x, w in zip((*got, g.q, g.k), (*want, *grads)):
            close(x, w)
        kept = big.clone()
        tcu.norm_rotate(q, k, rates, out=(q, k))
        assert torch.equal(q, got[0]) and torch.equal(k, got[1])
        assert torch.equal(big[..., 128 + extra:], kept[..., 128 + extra:])
        assert torch.equal(big[..., :extra], kept[..., :extra])


@gpu
@pytest.mark.parametrize("dtype", TYPES)
def test_rows_behind_the_last_sequence(tcu, dtype):
    nan = float("nan")
    a, dq, dk = inputs(dtype, (50,), 4, 2, 64, 32, offsets=offsets_of([10, 0, 20]))
    short = {n: v[:30] if n in ("q", "k") else v for n, v in a.items()}
    c, s, dq, dk = cuda(a), cuda(short), dq.cuda(), dk.cuda()
    for t in (c["q"], c["k"], dq, dk):
        t[30:] = nan
    out = (torch.full_like(c["q"], 7), torch.full_like(c["k"], 7))
    tcu.norm_rotate(**c, out=out)
    for got, want in zip(out, tcu.norm_rotate(**s)):
        assert torch.equal(got[:30], want) and (got[30:] == 7).all()
    g, w = tcu.norm_rotate_grad(dq, dk, **c), tcu.norm_rotate_grad(dq[:30], dk[:30], **s)
    for got, want in zip(g[:2], w[:2]):
        assert torch.equal(got[:30], want) and (got[30:] == 0).all()
    close(g.q_weight, w.q_weight.cpu().double())
    close(g.k_weight, w.k_weight.cpu().double())


@gpu
def test_nothing_to_do(tcu):
    for dtype in TYPES:
        q = torch.zeros(2, 0, 3, 8, dtype=dtype, device="cuda")
        rates, w = torch.ones(4, device="cuda"), torch.ones(8, device="cuda")
        y, z = tcu.norm_rotate(q, q, rates)
        assert y.shape == z.shape == q.shape
        g = tcu.norm_rotate_grad(q, q, q, q, rates, q_weight=w, k_weight=w)
        assert (g.q_weight == 0).all() and (g.k_weight == 0).all()
    # a head of zeros stays one
    q = torch.zeros(1, 2, 3, 8, device="cuda")
    assert (tcu.norm_rotate(q, q, rates)[0] == 0).all()


@gpu
def test_many_rows(tcu):
    """More rows than the card takes at once, against torch in 64 bits."""
    gen = torch.Generator(device="cuda").manual_seed(0)
    r = lambda *s: torch.randn(*s, generator=gen, device="cuda")  # noqa: E731
    q, k, dq, dk, w = r(3, 9001, 2, 16), r(3, 9001, 1, 16), r(3, 9001, 2, 16), r(3, 9001, 1, 16), r(16)
    rates = torch.rand(8, generator=gen, device="cuda")
    a = dict(q=q.cpu(), k=k.cpu(), rates=rates.cpu(), q_weight=w.cpu(), k_weight=w.cpu(),
             positions=None, offsets=None)
    outs, grads, weights = reference(a, 1e-6, False, dq.cpu(), dk.cpu())
    for got, want in zip(tcu.norm_rotate(q, k, rates, q_weight=w, k_weight=w), outs):
        close(got, want)
    g = tcu.norm_rotate_grad(dq, dk, q, k, rates, q_weight=w, k_weight=w)
    for got, want in zip(g, grads + weights):
        close(got, want)


@gpu
@pytest.mark.parametrize("interleaved", [False, True])
def test_autograd_and_differences(tcu, interleaved):
    a, dq, dk = inputs(torch.float32, (2, 5), 3, 1, 16, 6)
    c, dq, dk = cuda(a), dq.cuda(), dk.cuda()
    names = ("q", "k", "q_weight", "k_weight")
    leaves = {n: c[n].clone().requires_grad_() for n in names}
    y, z = tcu.norm_rotate(**{**c, **leaves}, interleaved=interleaved)
    # gradients arrive in any layout
    ((y.transpose(1, 2) * dq.transpose(1, 2)).sum() + (z * dk).sum()).backward()
    g = tcu.norm_rotate_grad(dq, dk, **c, interleaved=interleaved)
    gen = torch.Generator().manual_seed(5)
    for n in names:
        assert torch.equal(leaves[n].grad, getattr(g, n)), n
        way = randn(gen, *c[n].shape).cuda()

        def loss(h):
            y, z = tcu.norm_rotate(**dict(c, **{n: c[n] + h * way}), interleaved=interleaved)
            return ((y * dq).double().sum() + (z * dk).double().sum()).item()

        slope = (loss(1e-2) - loss(-1e-2)) / 2e-2  # h^2 of the third derivative, 2^-24 / h
        terms = getattr(g, n).double() * way.double()
        assert abs(slope - terms.sum().item()) <= 2e-3 * max(abs(terms.sum().item()), terms.norm().item())


@gpu
def test_graphs_and_streams(tcu):
    a, dq, dk = inputs(torch.bfloat16, (60,), 4, 2, 64, 32, offsets=offsets_of([30, 30]))
    c, dq, dk = cuda(a), dq.cuda(), dk.cuda()
    want, grads = tcu.norm_rotate(**c), tcu.norm_rotate_grad(dq, dk, **c)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    got = tcu.norm_rotate(**c, stream=side)
    torch.cuda.current_stream().wait_stream(side)
    assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        got, g = tcu.norm_rotate(**c), tcu.norm_rotate_grad(dq, dk, **c)
    for _ in range(2):
        for t in (*got, *g):
            t.fill_(3)
        graph.replay()
        torch.cuda.synchronize()
        for x, w in zip((*got, *g), (*want, *grads)):
            assert torch.equal(x, w)


# ------------------------------------------------------------ without a GPU
@pytest.mark.parametrize("interleaved", [False, True])
def test_reference_against_differences(interleaved):
    gen = torch.Generator().manual_seed(0)
    x, w = (torch.randn(*s, generator=gen, dtype=torch.float64).requires_grad_()
            for s in ((3, 2, 6), (6,)))
    rates, place = torch.rand(2, generator=gen, dtype=torch.float64), torch.tensor([0, 4, 9])
    assert torch.autograd.gradcheck(
        lambda x, w: ref.norm_rotate(x, w, rates, place, 1e-3, interleaved), (x, w))


def args(attn, **change):
    fake = 0x10000  # never dereferenced: every call here is refused
    r = attn._Rows(fake, 400, 80)
    v = dict(type=0, sequences=2, heads=4, kv_heads=2, dim=16, turned=8, eps=1e-6, rows=5,
             rates=fake, dq_weight=fake, workspace=fake, workspace_bytes=1 << 30,
             **{k: r for k in ("q", "k", "y_q", "y_k", "dy_q", "dy_k", "dq", "dk")})
    v.update(change)
    return attn._RotateArgs(**v)


INVALID, UNSUPPORTED = 1, 2


@pytest.mark.parametrize("call,change,status", [
    ("", dict(type=3), INVALID), ("", dict(dim=0), INVALID), ("", dict(dim=15), INVALID),
    ("", dict(dim=258), UNSUPPORTED), ("", dict(turned=0), INVALID), ("", dict(turned=9), INVALID),
    ("", dict(heads=0), INVALID), ("", dict(kv_heads=0), INVALID), ("", dict(rows=-1), INVALID),
    ("", dict(rows=2 ** 31), UNSUPPORTED), ("", dict(eps=-1.0), INVALID),
    ("", dict(eps=float("nan")), INVALID), ("", dict(rates=None), INVALID),
    ("", dict(q_weight=0x10001), INVALID), ("", dict(positions=0x10002), INVALID),
    ("", dict(heads=2 ** 21), UNSUPPORTED),
    ("_grad", dict(workspace_bytes=8), INVALID), ("_grad", dict(workspace=0x10002), INVALID),
    ("_grad", dict(dq_weight=0x10002), INVALID)])
def test_refusals(tcu, call, change, status):
    from paper_1908_06649_gb300 import attention as attn
    assert getattr(attn._lib(), "tcu_norm_rotate" + call)(args(attn, **change), None) == status


def test_refused_rows_and_workspaces(tcu):
    from paper_1908_06649_gb300 import attention as attn
    L = attn._lib()
    far, odd = attn._Rows(0x10000, 2 ** 33, 2 ** 31), attn._Rows(0x10001, 400, 80)
    for k in ("q", "k", "y_q", "y_k"):
        assert L.tcu_norm_rotate(args(attn, **{k: far}), None) == UNSUPPORTED
        assert L.tcu_norm_rotate(args(attn, **{k: odd}), None) == INVALID
    for k in ("dy_q", "dy_k", "dq", "dk"):
        assert L.tcu_norm_rotate_grad(args(attn, **{k: odd}), None) == INVALID
    assert L.tcu_norm_rotate(None, None) == INVALID
    assert L.tcu_norm_rotate_grad_workspace(args(attn)) > 0
    assert L.tcu_norm_rotate_grad_workspace(args(attn, dq_weight=None)) == 0
    assert L.tcu_norm_rotate_grad_workspace(args(attn, dim=3)) == -1


def test_declared_symbols_and_layout(tcu, tmp_path):
    import os
    import re
    import subprocess
    from paper_1908_06649_gb300 import _build, attention as attn
    text = re.sub(r"/\*.*?\*/", "", open(_build.ATTN_HDR).read(), flags=re.S)
    assert sorted(set(re.findall(r"\b(tcu_[a-z_]+)\s*\(", text))) == sorted(attn.SYMBOLS)
    src, exe = tmp_path / "p.c", tmp_path / "p"
    src.write_text('#include <stddef.h>\n#include <stdio.h>\n#include "tcu_attn.h"\n'
                   "int main(void) { typedef tcu_norm_rotate_args A; typedef tcu_window_attention_args B;"
                   "printf(\"%zu %zu %zu %zu %zu %zu\\n\", sizeof(A), offsetof(A, rates),"
                   "offsetof(A, workspace_bytes), sizeof(B), offsetof(B, lse), offsetof(B, num_slots));"
                   "return 0; }\n")
    subprocess.run(["gcc", "-std=c99", "-Wall", "-Werror", "-I", os.path.dirname(_build.ATTN_HDR),
                    str(src), "-o", str(exe)], check=True)
    a, b = attn._RotateArgs, attn._AttentionArgs
    got = subprocess.run([str(exe)], capture_output=True, text=True, check=True).stdout.split()
    assert list(map(int, got)) == [ctypes.sizeof(a), a.rates.offset, a.workspace_bytes.offset,
                                   ctypes.sizeof(b), b.lse.offset, b.num_slots.offset]


@gpu
def test_refusals_of_tensors(tcu):
    q, rates = torch.zeros(2, 5, 3, 8, device="cuda"), torch.ones(4, device="cuda")
    ok = dict(q=q, k=q, rates=rates)
    tcu.norm_rotate(**ok)
    for bad in (dict(q=q.cpu()), dict(q=q[0]), dict(k=q[:, :4]), dict(k=q.half()), dict(k=q[0]),
                dict(rates=rates.double()), dict(rates=torch.ones(5, device="cuda")),
                dict(rates=rates[:0]), dict(q_weight=rates), dict(eps=-1.0), dict(q=q[..., :7]),
                dict(positions=torch.zeros(2, 5, device="cuda")), dict(q=q.transpose(2, 3)),
                dict(positions=torch.zeros(5, dtype=torch.int32, device="cuda")),
                dict(out=(q[:, :, :2], q)), dict(out=(q, q)), dict(k=None),
                dict(rates=rates.clone().requires_grad_())):
        with pytest.raises((ValueError, TypeError)):
            tcu.norm_rotate(**{**ok, **bad})
    with pytest.raises(ValueError):
        tcu.norm_rotate(q.clone().requires_grad_(), q, rates, out=(q, q.clone()))
    # the keys of one buffer over the queries' memory
    x = torch.zeros(4, 8, 8, device="cuda")
    place = torch.zeros(4, dtype=torch.int32, device="cuda")
    with pytest.raises(ValueError):
        tcu.norm_rotate(x[:, :3], x[:, 3:5], rates, positions=place, out=(x[:, 2:5], x[:, 5:7]))
    from torch.autograd import forward_ad
    with forward_ad.dual_level():
        dual = forward_ad.make_dual(q, torch.ones_like(q))
        for call in (lambda: tcu.norm_rotate(dual, q, rates),
                     lambda: tcu.norm_rotate_grad(q, dual, q, q, rates)):
            with pytest.raises(ValueError, match="forward-mode"):
                call()


@gpu
def test_beyond_32_bits_of_elements(tcu):
    rows = 270000
    gen = torch.Generator(device="cuda").manual_seed(0)
    q = torch.empty(1, rows, 64, 128, dtype=torch.bfloat16, device="cuda").normal_(generator=gen)
    k = q[:, :, :1].clone()
    rates = 10000.0 ** (-torch.arange(64, device="cuda") / 64)
    place = torch.arange(rows, dtype=torch.int32, device="cuda")
    y, z = tcu.norm_rotate(q, k, rates)
    end = [t[0, -100:].clone() for t in (q, k)]
    y2, z2 = tcu.norm_rotate(*end, rates, positions=place[-100:])
    assert torch.equal(y[0, -100:], y2) and torch.equal(z[0, -100:], z2)
    g = tcu.norm_rotate_grad(q, k, q, k, rates)
    w = tcu.norm_rotate_grad(*end, *end, rates, positions=place[-100:])
    assert torch.equal(g.q[0, -100:], w.q) and torch.equal(g.k[0, -100:], w.k)
