"""The sequence operators on the GPU at the limits of what they take."""
import pytest
import torch

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def pkg():
    from paper_1908_06649_gb300 import _build
    _build.build()
    import paper_1908_06649_gb300 as p
    p.lib()
    return p


def test_as_many_rows_as_there_can_be(pkg):
    """One channel of 2^31 - 4097 rows, its inputs one row broadcast: every
    row of y is written and, the state being forgotten within a few rows (a
    decay of e^-2 each), all but the first are the same to the bit."""
    rows = 2 ** 31 - 4097

    def same(*tail):
        return torch.full((1, 1) + tail, 1.0, dtype=torch.float16, device="cuda").expand(
            1, rows, *tail)

    A = torch.full((1, 1), -2.0, device="cuda")
    out = torch.full((1, rows, 1), float("nan"), dtype=torch.float16, device="cuda")
    _, last = pkg.state_scan(same(1), same(1), A, same(1, 1), same(1, 1), out=out)
    y = out.view(-1)
    # h = e^-2 h + 1
    want = 1 / (1 - float(torch.exp(torch.tensor(-2.0, dtype=torch.float64))))
    assert abs(float(last) - want) <= 1e-5 * want
    steady = torch.tensor(want, dtype=torch.float16, device="cuda")
    assert (y[:64] - steady).abs().max() < 0.2 and y[0] == 1
    part = 2 ** 28
    for first in range(64, rows, part):
        assert (y[first:first + part] == steady).all()


def test_long_sums_of_parameter_gradients(pkg):
    """Gradients of skip and dt_bias over 2^17 rows that are not split (160
    sequences fill the card), all terms the same 0.7: a decay of e^-1000 leaves
    q u = 0.7 of each row for the one, (C q B) u for the other.  A lane's sum goes
    in two levels, 16 terms and then their 1024 sums; three exchanges between
    lanes and 28 steps over sequences follow.  Each step rounds by 2^-24 at most."""
    rows, seqs = 2 ** 17, 160
    one = torch.ones(1, 1, 1, device="cuda").expand(seqs, rows, 1)
    u = torch.full((1, 1, 1), 0.7, device="cuda").expand(seqs, rows, 1)
    A = torch.full((1, 1), -1000.0, device="cuda")
    skip, bias = torch.ones(1, device="cuda"), torch.zeros(1, device="cuda")
    BC = one.unsqueeze(-1)
    _, _, marks = pkg.state_scan(u, one, A, BC, BC, skip=skip, dt_bias=bias, marks=True)
    g = pkg.state_scan_grad(one, u, one, A, BC, BC, skip=skip, dt_bias=bias, marks=marks)
    want = float(u[0, 0, 0].double()) * rows * seqs
    bound = (16 + rows // 128 + 3 + 28) * 2.0 ** -24 * want
    assert abs(float(g.skip) - want) <= bound
    assert abs(float(g.dt_bias) - want) <= bound
    assert float(g.A) == 0 and (g.dt == u).all() and (g.B == u[..., None]).all()


def test_strides_that_step_over_nothing(pkg):
    """One row, or one entry of a token call, may lie at any pitch: it is never
    taken a step.  (The token of one long sequence is a slice of this kind.)"""
    gen = torch.Generator(device="cuda").manual_seed(0)
    c, n, far = 40, 16, 2 ** 33 + 8
    randn = lambda *s: torch.randn(*s, generator=gen, device="cuda")  # noqa: E731
    u, dt, gate = randn(1, 1, c), randn(1, 1, c), randn(1, 1, c)
    A, B, C, w = -randn(c, n).abs(), randn(1, 1, 1, n), randn(1, 1, 1, n), randn(c, 4)
    apart = lambda t: t.as_strided(t.shape, (far, far) + t.stride()[2:])  # noqa: E731
    state, past = randn(1, c, n), randn(1, 3, c)

    def scan(f):
        args = f(u), f(dt), A, f(B), f(C)
        y, last, marks = pkg.state_scan(*args, gate=f(gate), state=state, marks=True)
        g = pkg.state_scan_grad(f(u), *args, gate=f(gate), state=state, marks=marks)
        return [y, last] + [v for v in g if v is not None]

    def conv(f):
        g = pkg.short_conv_grad(f(dt), f(u), w, state=past)
        return list(pkg.short_conv(f(u), w, state=past)) + [v for v in g if v is not None]

    def token(f):
        cache, rows = state.clone(), past.clone()
        one = lambda t: f(t)[:, 0]  # noqa: E731
        y = pkg.state_scan_step(one(u), one(dt), A, one(B), one(C), cache, gate=one(gate),
                                out=f(torch.empty_like(u))[:, 0])
        return [y, cache, pkg.short_conv_step(one(u), rows, w), rows]

    for call in (scan, conv, token):
        for got, want in zip(call(apart), call(lambda t: t)):
            assert torch.equal(got, want)
