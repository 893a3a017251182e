"""The recurrence and attention operators run together, as the example of them
does: serving against whole prompts, and gradients against the definitions in
64 bits; bounds set before the first run."""
import importlib.util
import math
import os

import pytest
import torch

import mixing_reference as ref
import sequence_reference as seq

pytestmark = pytest.mark.gpu
HERE = os.path.dirname(os.path.abspath(__file__))


@pytest.fixture(scope="module")
def example():
    from paper_1908_06649_gb300 import _build
    _build.build()
    path = os.path.join(os.path.dirname(HERE), "examples", "local_block.py")
    spec = importlib.util.spec_from_file_location("local_block", path)
    m = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(m)
    return m


def test_tokens_continue_packed_prompts(example):
    """bf16 throughout: eight roundings of 2^-8 on the way to an output."""
    assert example.serve(example.Block()) <= 8 * 2.0 ** -8


def test_it_trains(example):
    first, last = example.train(example.Block(), steps=3)
    assert math.isfinite(first) and math.isfinite(last)


def of_definitions(block, x, offsets):
    """The block from the definitions, in 64 bits."""
    p = [t.detach().cpu().double().requires_grad_() for t in block.parameters()]
    w_in, w_mid, w_qkv, w_out, taps, log_rate, q_weight, k_weight = p
    rates, h, kv, d = block.rates.cpu().double(), block.heads, block.kv_heads, block.dim
    v, f, a = (x @ w_in).chunk(3, -1)
    u, _ = seq.conv(v, taps, act=True, offsets=offsets)
    y, _ = ref.gated(u, f, a, log_rate.exp(), offsets=offsets)
    z = x + y @ w_mid
    q, k, v = (z @ w_qkv).unflatten(-1, (h + 2 * kv, d)).split([h, kv, kv], -2)
    place = ref.positions_of(q, offsets)
    q, k = (ref.norm_rotate(t, w, rates, place, 1e-6, False) for t, w in ((q, q_weight), (k, k_weight)))
    y, _ = ref.attention(q, k, v, offsets=offsets, **block.seen)
    return z + y.flatten(-2) @ w_out, p


@pytest.mark.parametrize("packed", [False, True])
def test_gradients(example, packed):
    """A dozen roundings of at most 2^-8 of what they round lie on the way to an
    output and back to a parameter, their errors of random sign: their root sum
    of squares is 3.5 2^-8, held to 6 2^-8."""
    block = example.Block()
    gen = torch.Generator().manual_seed(3)
    off = ref.offsets_of([40, 0, 25, 5]) if packed else None
    x = torch.randn(*((70,) if packed else (2, 35)), 128, generator=gen).bfloat16()
    dy = torch.randn(*x.shape, generator=gen).bfloat16()
    leaf = x.double().requires_grad_()
    want, p = of_definitions(block, leaf, off)
    grads = torch.autograd.grad(want, [leaf, *p], dy.double())
    mine = x.cuda().requires_grad_()
    out, _, _ = block.prompt(mine, None if off is None else off.cuda())
    out.backward(dy.cuda())

    def near(got, exact, name):
        far = (got.cpu().double() - exact).norm() / exact.norm()
        assert far <= 6 * 2.0 ** -8, (name, float(far))

    near(out.detach(), want.detach(), "out")
    names = ("w_in", "w_mid", "w_qkv", "w_out", "taps", "log_rate", "q_weight", "k_weight")
    for name, got, exact in zip(("x", *names), (mine, *block.parameters()), grads):
        near(got.grad, exact, name)
