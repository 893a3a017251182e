"""The gated recurrence where states are not finite."""
import pytest
import torch

import mixing_reference as ref
from mixing_reference import TYPES, close, cuda, offsets_of, randn

gpu = pytest.mark.gpu


@pytest.fixture(scope="module")
def tcu():
    from paper_1908_06649_gb300 import _build
    _build.build()
    import paper_1908_06649_gb300 as p
    p.lib()
    return p


@gpu
@pytest.mark.parametrize("bad", [float("inf"), -float("inf"), float("nan")])
@pytest.mark.parametrize("channels", [6, 64 * 20])  # blocks of a cluster, blocks alone
def test_what_is_not_finite_stays_in_its_sequence(tcu, bad, channels):
    """Decays whose product over a warp's rows, or a tile's, is below fp32's
    range end no sequence: a state, an input or a gradient that is not finite
    reaches every later (earlier) row of its own sequence, packed as dense, and
    no other."""
    gen = torch.Generator().manual_seed(0)
    lengths = [50, 700, 60]
    off = offsets_of(lengths).cuda()
    x, dy = randn(gen, 2, sum(lengths), channels).cuda().unbind(0)
    open_ = torch.full_like(x, 8.0)
    rate = torch.linspace(0.05, 30, channels).cuda()
    state, dlast = randn(gen, 2, 3, channels).cuda().unbind(0)
    args = (open_, open_, rate)
    clean, end, marks = tcu.gated_scan(x, *args, state=state, offsets=off, marks=True)
    g = tcu.gated_scan_grad(dy, x, *args, marks=marks, state=state, offsets=off, dlast=dlast)
    for where in ("state", "x"):
        x2, state2 = x.clone(), state.clone()
        if where == "state":
            state2[1] = bad
        else:
            x2[53] = bad
        y, last, _ = tcu.gated_scan(x2, *args, state=state2, offsets=off, marks=True)
        assert torch.equal(y[:50], clean[:50]) and torch.equal(y[750:], clean[750:]), where
        assert not y[53:750].isfinite().any(), where
        assert torch.equal(last[::2], end[::2]) and not last[1].isfinite().any()
        alone, _ = tcu.gated_scan(x2[None, 50:750], open_[None, 50:750], open_[None, 50:750], rate,
                                  state=state2[1:2])
        assert not alone[:, 3:].isfinite().any()
    for where in ("dlast", "dy"):
        dy2, dlast2 = dy.clone(), dlast.clone()
        if where == "dlast":
            dlast2[1] = bad
        else:
            dy2[747] = bad
        b = tcu.gated_scan_grad(dy2, x, *args, marks=marks, state=state, offsets=off, dlast=dlast2)
        assert torch.equal(b.x[:50], g.x[:50]) and torch.equal(b.x[750:], g.x[750:]), where
        assert not b.x[50:748].isfinite().any(), where
        assert torch.equal(b.state[::2], g.state[::2]) and not b.state[1].isfinite().any()
