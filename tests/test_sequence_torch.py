"""The sequence operators as citizens of torch: no channels, in-place writes
that autograd has to know of, forward mode, streams, first use by threads."""
import threading

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


@pytest.mark.gpu
def test_caches_that_record_a_gradient(seq):
    """A token call has no gradient: a cache or an output that would need one is
    refused, as every other argument is; under no_grad it is advanced."""
    a, state = tokens()
    w, x = torch.randn(16, 4, device="cuda"), a["u"]
    _, past = seq.short_conv(torch.randn(4, 6, 16, device="cuda"), w.clone().requires_grad_())
    assert past.requires_grad
    with pytest.raises(ValueError):
        seq.short_conv_step(x, past, w)
    with pytest.raises(ValueError):
        seq.state_scan_step(**a, state=state.clone().requires_grad_())
    for make in (lambda out: seq.short_conv_step(x, past.detach().clone(), w, out=out),
                 lambda out: seq.state_scan_step(**a, state=state.clone(), out=out),
                 lambda out: seq.short_conv(x[None], w, out=out[None]),
                 lambda out: seq.state_scan(x[None], a["dt"][None], a["A"], a["B"][None],
                                            a["C"][None], out=out[None])):
        with pytest.raises(ValueError):
            make(torch.zeros_like(x).requires_grad_())
        with torch.no_grad():
            make(torch.zeros_like(x).requires_grad_())
    with torch.no_grad():
        before = past.clone()
        seq.short_conv_step(x, past, w)
        assert torch.equal(past[:, :2], before[:, 1:]) and torch.equal(past[:, 2], x)


@pytest.mark.gpu
def test_writes_in_place_are_known_to_autograd(seq):
    """What an operation has saved for its backward pass may not change under it:
    as torch's own in-place operations, the calls raise the tensor's version."""
    a, state = tokens()
    w, x = torch.randn(16, 4, device="cuda"), a["u"]
    past = torch.randn(4, 3, 16, device="cuda")
    prompt = (x[None], a["dt"][None], a["A"], a["B"][None], a["C"][None])
    out = torch.zeros_like(x)
    for t, call in ((past, lambda: seq.short_conv_step(x, past, w)),
                    (state, lambda: seq.state_scan_step(**a, state=state)),
                    (out, lambda: seq.short_conv_step(x, past, w, out=out)),
                    (out, lambda: seq.state_scan_step(**a, state=state, out=out)),
                    (out, lambda: seq.short_conv(x[None], w, out=out[None])),
                    (out, lambda: seq.state_scan(*prompt, out=out[None]))):
        p = torch.ones_like(t).requires_grad_()
        loss = (p * t).sum()  # saves t
        seen = t._version
        call()
        assert t._version > seen
        with pytest.raises(RuntimeError, match="modified by an inplace operation"):
            loss.backward()
    # inference tensors have no version, and serve as before
    with torch.inference_mode():
        cache, to = state.clone(), torch.zeros_like(x)
        seq.state_scan_step(**a, state=cache, out=to)
    seq.state_scan_step(**a, state=cache, out=to)


def every_call(seq, a, state, wrap):
    """(argument, call) for each argument of each call, wrapped alone."""
    x, w = a["u"], torch.randn(16, 4, device=a["u"].device)
    past = torch.randn(4, 3, 16, device=x.device)
    rows = {k: v[None] if k in ("u", "dt", "B", "C") else v for k, v in a.items()}
    marks = torch.zeros(1, 1, 16, 8, device=x.device)
    own = state[:1]

    def with_one(call, args):
        for k in args:
            if args[k] is not None:
                yield k, lambda k=k: call(**dict(args, **{k: wrap(args[k])}))

    yield from with_one(seq.short_conv, dict(x=x[None], weight=w, state=past[:1]))
    yield from with_one(seq.short_conv_grad,
                        dict(dy=x[None], x=x[None], weight=w, state=past[:1], dlast=past[:1]))
    yield from with_one(seq.short_conv_step, dict(x=x, state=past, weight=w))
    yield from with_one(seq.state_scan, dict(rows, gate=rows["u"], state=own))
    yield from with_one(seq.state_scan_grad, dict(rows, dy=rows["u"], marks=marks, gate=rows["u"],
                                                  state=own, dlast=own))
    yield from with_one(seq.state_scan_step, dict(a, state=state, gate=a["u"]))


def forward_mode(seq, a, state):
    from torch.autograd import forward_ad
    with forward_ad.dual_level():
        count = 0
        for k, call in every_call(seq, a, state,
                                  lambda t: forward_ad.make_dual(t, torch.ones_like(t))):
            with pytest.raises(ValueError, match="forward-mode"):
                call()
            count += 1
    assert count > 30
    return count


def test_forward_mode_is_refused(seq):
    """Before anything else is looked at, the device included."""
    gen = torch.Generator().manual_seed(0)
    r = lambda *s: torch.randn(*s, generator=gen)  # noqa: E731
    forward_mode(seq, dict(u=r(4, 16), dt=r(4, 16), A=-r(16, 8).abs(), B=r(4, 8), C=r(4, 8)),
                 r(4, 16, 8))


@pytest.mark.gpu
def test_forward_mode_on_the_gpu(seq):
    """A tangent would be lost without a word; without one, a dual level is
    nothing to the calls."""
    from torch.autograd import forward_ad
    a, state = tokens()
    forward_mode(seq, a, state)
    want = seq.state_scan_step(**a, state=state.clone())
    with forward_ad.dual_level():
        assert torch.equal(seq.state_scan_step(**a, state=state.clone()), want)


class FakeStream:
    cuda_stream = 0

    def __init__(self, index):
        self.device = torch.device("cuda", index)


def test_a_stream_of_another_device_is_refused(seq):
    """Its kernels would start on that device, on memory of this one.  Nothing
    is entered or launched: no GPU is needed to be refused."""
    with pytest.raises(ValueError, match="cuda:1"):
        seq._On(0, FakeStream(1))
    seq._On(1, FakeStream(1))


@pytest.mark.gpu
def test_a_stream_of_another_device_is_refused_by_every_call(seq):
    a, state = tokens()
    x, w, other = a["u"], torch.randn(16, 4, device="cuda"), FakeStream(1)
    rows = [a[k][None] if k != "A" else a[k] for k in ("u", "dt", "A", "B", "C")]
    marks = seq.state_scan(*rows, marks=True)[2]
    before = state.clone()
    for call in (lambda: seq.short_conv(x[None], w, stream=other),
                 lambda: seq.short_conv_grad(x[None], x[None], w, stream=other),
                 lambda: seq.short_conv_step(x, torch.zeros(4, 3, 16, device="cuda"), w, stream=other),
                 lambda: seq.state_scan(*rows, stream=other),
                 lambda: seq.state_scan_grad(x[None], *rows, marks=marks, stream=other),
                 lambda: seq.state_scan_step(**a, state=state, stream=other)):
        with pytest.raises(ValueError, match="cuda:1"):
            call()
    assert torch.equal(state, before) and torch.cuda.current_device() == 0


def test_entries_are_published_with_their_types(seq, monkeypatch):
    """A second thread whose first call falls into the binding finds either no
    entry or a finished one: an entry without types takes a stream's address
    for a 32-bit number.  Here the other thread looks after every step of it."""
    class Entry:
        def __init__(self):
            self.__dict__["types"] = set()

        def __setattr__(self, name, value):
            look()
            self.types.add(name)
            look()

    class Library:
        def __init__(self):
            self.named = {}

        def __getattr__(self, name):
            if not name.startswith("tcu_"):
                raise AttributeError(name)
            return self.named.setdefault(name, Entry())

        def __getitem__(self, name):
            return Entry()

    def look():
        for name, f in dict(seq._calls).items():
            assert f.types == {"argtypes", "restype"}, name

    monkeypatch.setattr(seq, "_bound", None)
    monkeypatch.setattr(seq, "_calls", {})
    monkeypatch.setattr(seq, "lib", Library)
    first = seq._lib()
    look()
    assert sorted(seq._calls) == sorted(seq.SYMBOLS) and seq._lib() is first


def test_threads_share_one_binding(seq, monkeypatch):
    real, made = seq.lib, []

    def slow():
        made.append(1)
        started.wait(2)
        return real()

    started, got = threading.Event(), []
    monkeypatch.setattr(seq, "_bound", None)
    monkeypatch.setattr(seq, "_calls", {})
    monkeypatch.setattr(seq, "lib", slow)
    threads = [threading.Thread(target=lambda: got.append(seq._lib())) for _ in range(4)]
    for t in threads:
        t.start()
    started.set()
    for t in threads:
        t.join()
    assert len(made) == 1 and len(got) == 4 and all(g is got[0] for g in got)
