"""Angles of far positions and large rates, against integer arithmetic."""
import math
from fractions import Fraction

import pytest
import torch

gpu = pytest.mark.gpu
FAR = [1, -1, 1000, 10 ** 6 + 3, 2 ** 30 + 12345, 2 ** 31 - 1, -2 ** 31]


@pytest.fixture(scope="module")
def tcu():
    from paper_1908_06649_gb300 import _build
    _build.build()
    import paper_1908_06649_gb300 as p
    p.lib()
    return p


def over_two_pi(bits=400):
    """1 / (2 pi) as a fraction, pi by Machin's formula."""
    one = 1 << bits

    def arctan(n):
        total, term, k = 0, one // n, 1
        while term:
            total += term // k if k % 4 == 1 else -(term // k)
            term //= n * n
            k += 2
        return total

    return Fraction(one, 2 * (16 * arctan(5) - 4 * arctan(239)))


def angles(positions, rates):
    """cos and sin of position x rate, its whole turns taken off exactly."""
    turn = over_two_pi()
    turns = [[float(p * Fraction(r) * turn % 1) for r in rates] for p in positions]
    t = torch.tensor(turns, dtype=torch.float64) * (2 * math.pi)
    return torch.cos(t), torch.sin(t)


def rates_of(n):
    gen = torch.Generator().manual_seed(0)
    small = 10000.0 ** (-torch.arange(n) / n)
    large = torch.randn(n, generator=gen) * 30
    wide = torch.logspace(-3, math.log10(2.0 ** 32), n) * torch.where(torch.arange(n) % 2 == 0, 1, -1)
    return small, large, wide.float()


@gpu
@pytest.mark.parametrize("interleaved", [False, True])
def test_angles(tcu, interleaved):
    """Heads of (1, 0) pairs come out as sqrt(2) cos and sqrt(2) sin.  An angle is
    2^-26 turns off by its rounding to fp32 and 2^-31 by what a position
    multiplies, 1.0e-7 in radians; sine and cosine of fp32 are two steps off,
    1.2e-7; the norm, its reciprocal root and the products six roundings of
    2^-24: sqrt(2) of 5.8e-7 in all."""
    n = 64
    place = torch.tensor(FAR, dtype=torch.int32).cuda()
    one, zero = torch.ones(len(FAR), 1, n), torch.zeros(len(FAR), 1, n)
    q = (torch.stack([one, zero], -1).flatten(-2) if interleaved else torch.cat([one, zero], -1)).cuda()
    for rates in rates_of(n):
        y, _ = tcu.norm_rotate(q, q, rates.cuda(), positions=place, eps=0.0, interleaved=interleaved)
        cos, sin = angles(FAR, rates.tolist())
        got = y[:, 0].cpu().double()
        c, s = (got[:, ::2], got[:, 1::2]) if interleaved else got.split(n, -1)
        assert (c - cos * 2 ** 0.5).abs().max() <= 8.3e-7
        assert (s - sin * 2 ** 0.5).abs().max() <= 8.3e-7
        # against the angles back again: dy of (cos, sin) pairs gives d of (1, 0)
        # of the normed values; n = sqrt(2) (1, 0) is orthogonal to it but for
        # its own direction, which the norm's gradient takes off: pairs of (0, 1)
        turned = torch.stack([-sin, cos], -1).flatten(-2) if interleaved else torch.cat([-sin, cos], -1)
        g = tcu.norm_rotate_grad(turned.float()[:, None].cuda(), torch.zeros_like(q), q, q, rates.cuda(),
                                 positions=place, eps=0.0, interleaved=interleaved)
        back = g.q[:, 0].cpu().double() / 2 ** 0.5
        a, b = (back[:, ::2], back[:, 1::2]) if interleaved else back.split(n, -1)
        assert a.abs().max() <= 8.3e-7 and (b - 1).abs().max() <= 8.3e-7


@gpu
@pytest.mark.parametrize("bad", [float("nan"), float("inf"), -float("inf")])
@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("dim", [128, 18, 6])
def test_rates_that_are_no_numbers(tcu, bad, interleaved, dim):
    """Their pairs come out as no numbers, the others as they were."""
    n = dim // 2 - 1
    gen = torch.Generator().manual_seed(0)
    q, dq = torch.randn(2, 5, 3, 2, dim, generator=gen).cuda().unbind(0)
    rates = torch.rand(n, generator=gen).cuda()
    place = torch.tensor([0, 1, -4, 70000, 2 ** 31 - 1], dtype=torch.int32).cuda()[:, None].repeat(1, 3)
    want, _ = tcu.norm_rotate(q, q, rates, positions=place, interleaved=interleaved)
    rates[n - 1] = bad
    got, _ = tcu.norm_rotate(q, q, rates, positions=place, interleaved=interleaved)
    g = tcu.norm_rotate_grad(dq, dq, q, q, rates, positions=place, interleaved=interleaved)
    gone = torch.zeros(dim, dtype=torch.bool)
    gone[[2 * n - 2, 2 * n - 1] if interleaved else [n - 1, 2 * n - 1]] = True
    assert got[..., gone].isnan().all() and torch.equal(got[..., ~gone], want[..., ~gone])
    assert g.q[..., gone].isnan().all()


def test_reference():
    assert abs(float(over_two_pi()) - 1 / (2 * math.pi)) < 1e-17
    cos, sin = angles([0, 3, -2], [0.5, 2.0])
    t = torch.tensor([[0, 0], [1.5, 6], [-1, -4]], dtype=torch.float64)
    assert torch.allclose(cos, torch.cos(t)) and torch.allclose(sin, torch.sin(t))
