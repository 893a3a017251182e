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
