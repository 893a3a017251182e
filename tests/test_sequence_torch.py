"""The sequence operators as citizens of torch: no channels, in-place writes
that autograd has to know of, forward mode, streams, first use by threads."""
import threading
import types

import pytest
import torch


@pytest.fixture(scope="module")
def seq():
    from paper_1908_06649_gb300 import _build
    _build.build()
    from paper_1908_06649_gb300 import sequence
    return sequence


def tokens(b=4, c=16, n=8):
    gen = torch.Generator().manual_seed(0)
    r = lambda *s: torch.randn(*s, generator=gen).cuda()  # noqa: E731
    return dict(u=r(b, c), dt=r(b, c), A=-r(c, n).abs(), B=r(b, n), C=r(b, n)), r(b, c, n)


@pytest.mark.gpu
@pytest.mark.parametrize("packed", [False, True])
def test_gradients_of_no_channels_are_zeros(seq, packed):
    """Sums over no channels; freed memory full of NaN lies ready to be handed out."""
    lead, seqs, n = ((12,) if packed else (2, 6)), 2, 4
    off = torch.tensor([0, 5, 12], dtype=torch.int32, device="cuda") if packed else None
    u = torch.zeros(*lead, 0, device="cuda")
    A = torch.zeros(0, n, device="cuda")
    B, C = (torch.randn(*lead, 3, n, device="cuda") for _ in range(2))
    y, last, marks = seq.state_scan(u, u, A, B, C, marks=True, offsets=off)
    assert y.shape == u.shape and last.shape == (seqs, 0, n)
    spoiled = [torch.full_like(B, float("nan")) for _ in range(8)]
    del spoiled
    g = seq.state_scan_grad(u, u, u, A, B, C, marks=marks, offsets=off)
    assert g.B.shape == B.shape and (g.B == 0).all() and (g.C == 0).all()
    assert g.u.shape == u.shape and g.A.shape == A.shape
