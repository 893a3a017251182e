"""The sequence operators without a GPU: the C boundary (include/tcu_seq.h),
its refusals before any launch, and the 64-bit definitions the GPU tests
compare with, against differences."""
import ctypes
import os
import re
import subprocess

import pytest
import torch

import sequence_reference as ref
from paper_1908_06649_gb300 import _build

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
HEADER = os.path.join(ROOT, "include", "tcu_seq.h")


@pytest.fixture(scope="module")
def seq():
    _build.build()
    from paper_1908_06649_gb300 import sequence
    return sequence


def test_declared_symbols_are_exported(seq):
    src = re.sub(r"/\*.*?\*/", "", open(HEADER).read(), flags=re.S)
    names = sorted(set(re.findall(r"\b(tcu_[a-z_]+)\s*\(", src)))
    assert names == sorted(seq.SYMBOLS)
    _build.build(checked=True)
    for path in (_build.LIB_PATH, _build.CHECKED_LIB_PATH):
        out = subprocess.run(["nm", "-D", "--defined-only", path], capture_output=True, text=True,
                             check=True).stdout
        exported = set(re.findall(r"\bT (\w+)", out))
        assert set(names) <= exported


C_PROGRAM = r"""
#include <stddef.h>
#include <stdio.h>
#include "tcu_seq.h"
int main(void) {
  tcu_short_conv_args c = {0};
  tcu_state_scan_args s = {0};
  printf("%zu %zu %zu %zu %zu %zu\n", sizeof c, offsetof(tcu_short_conv_args, weight),
         offsetof(tcu_short_conv_args, num_slots), sizeof s, offsetof(tcu_state_scan_args, A),
         offsetof(tcu_state_scan_args, num_slots));
  if (tcu_short_conv(NULL, NULL) != TCU_DFT_ERR_INVALID) return 1;
  if (tcu_state_scan(&s, NULL) != TCU_DFT_ERR_INVALID) return 2;
  c.width = 4; c.channels = 8; c.sequences = 1; c.rows = 3;
  if (tcu_short_conv(&c, NULL) != TCU_DFT_ERR_INVALID) return 3;
  c.width = TCU_SEQ_MAX_WIDTH + 1;
  if (tcu_short_conv(&c, NULL) != TCU_DFT_ERR_UNSUPPORTED) return 4;
  return 0;
}
"""


def test_c_program_and_struct_layout(seq, tmp_path):
    src, exe = tmp_path / "p.c", tmp_path / "p"
    src.write_text(C_PROGRAM)
    subprocess.run(["gcc", "-std=c99", "-Wall", "-Werror", "-I", os.path.dirname(HEADER), str(src),
                    "-o", str(exe), _build.LIB_PATH, "-Wl,-rpath," + os.path.dirname(_build.LIB_PATH)],
                   check=True)
    out = subprocess.run([str(exe)], capture_output=True, text=True)
    assert out.returncode == 0, out
    got = list(map(int, out.stdout.split()))
    c, s = seq._ConvArgs, seq._ScanArgs
    assert got == [ctypes.sizeof(c), c.weight.offset, c.num_slots.offset, ctypes.sizeof(s),
                   s.A.offset, s.num_slots.offset]


def conv_args(seq, **change):
    fake = 0x10000  # never dereferenced: every call here is refused
    v = dict(type=0, width=4, sequences=2, rows=5, channels=8, x=seq._Rows(fake, 40, 8),
             y=seq._Rows(fake, 40, 8), dy=seq._Rows(fake, 40, 8), dx=seq._Rows(fake, 40, 8),
             weight=fake, dweight=fake, last=fake, workspace=fake, workspace_bytes=1 << 30)
    v.update(change)
    return seq._ConvArgs(**v)


def scan_args(seq, **change):
    fake = 0x10000
    r = seq._Rows(fake, 40, 8)
    v = dict(type=0, sequences=2, groups=1, rows=5, channels=8, states=16, A=fake, dA=fake,
             marks=fake, last=fake, workspace=fake, workspace_bytes=1 << 30,
             **{k: r for k in ("u", "dt", "y", "B", "C", "dy", "du", "ddt", "dB", "dC")})
    v.update(change)
    return seq._ScanArgs(**v)


INVALID, UNSUPPORTED = 1, 2


@pytest.mark.parametrize("call,change,status", [
    ("tcu_short_conv", dict(type=3), INVALID), ("tcu_short_conv", dict(width=0), INVALID),
    ("tcu_short_conv", dict(width=9), UNSUPPORTED), ("tcu_short_conv", dict(rows=-1), INVALID),
    ("tcu_short_conv", dict(rows=2 ** 31), UNSUPPORTED),
    ("tcu_short_conv", dict(channels=0), INVALID), ("tcu_short_conv", dict(weight=None), INVALID),
    ("tcu_short_conv", dict(weight=0x10002), INVALID), ("tcu_short_conv", dict(bias=0x10001), INVALID),
    ("tcu_short_conv", dict(last=0x10002), INVALID),
    ("tcu_short_conv_grad", dict(dweight=None), INVALID),
    ("tcu_short_conv_grad", dict(workspace_bytes=16), INVALID),
    ("tcu_short_conv_step", dict(), INVALID),
    ("tcu_short_conv_step", dict(rows=1, num_slots=1), INVALID),
    ("tcu_short_conv_step", dict(rows=1, num_slots=2, last=None), INVALID)])
def test_conv_refusals(seq, call, change, status):
    assert getattr(seq._lib(), call)(conv_args(seq, **change), None) == status


@pytest.mark.parametrize("call,change,status", [
    ("tcu_state_scan", dict(type=-1), INVALID), ("tcu_state_scan", dict(states=0), INVALID),
    ("tcu_state_scan", dict(states=129), UNSUPPORTED),
    ("tcu_state_scan", dict(groups=3), INVALID), ("tcu_state_scan", dict(groups=0), INVALID),
    ("tcu_state_scan", dict(rows=2 ** 31), UNSUPPORTED), ("tcu_state_scan", dict(A=None), INVALID),
    ("tcu_state_scan", dict(state=0x10002), INVALID),
    ("tcu_state_scan", dict(offsets=0x10000, workspace_bytes=0), INVALID),
    ("tcu_state_scan_grad", dict(marks=None), INVALID),
    ("tcu_state_scan_grad", dict(dA=None), INVALID),
    ("tcu_state_scan_grad", dict(workspace_bytes=64), INVALID),
    ("tcu_state_scan_step", dict(), INVALID),
    ("tcu_state_scan_step", dict(rows=1, num_slots=1), INVALID)])
def test_scan_refusals(seq, call, change, status):
    a = scan_args(seq, **change)
    for row in ("u", "dt"):
        if change.get(row):
            setattr(a, row, change[row])
    assert getattr(seq._lib(), call)(a, None) == status


def test_workspaces_need_no_gpu(seq):
    L = seq._lib()
    assert L.tcu_short_conv_grad_workspace(conv_args(seq)) > 0
    assert L.tcu_short_conv_grad_workspace(conv_args(seq, width=9)) == -1
    assert L.tcu_state_scan_grad_workspace(scan_args(seq)) > 0
    assert L.tcu_state_scan_workspace(scan_args(seq, states=500)) == -1


def test_tensors_off_the_gpu_are_refused(seq):
    import paper_1908_06649_gb300 as pkg
    x, w = torch.zeros(2, 5, 8), torch.zeros(8, 4)
    with pytest.raises(ValueError):
        pkg.short_conv(x, w)
    with pytest.raises(ValueError):
        pkg.state_scan(x, x, torch.zeros(8, 16), torch.zeros(2, 5, 16), torch.zeros(2, 5, 16))
    with pytest.raises(TypeError):
        pkg.short_conv(None, w)
    with pytest.raises(AttributeError):
        pkg.no_such_operator


# ---- the reference itself
def _randn(gen, *shape):
    return torch.randn(*shape, generator=gen, dtype=torch.float64).requires_grad_()


@pytest.mark.parametrize("packed", [False, True])
def test_reference_gradients_against_differences(packed):
    gen = torch.Generator().manual_seed(0)
    off = torch.tensor([0, 2, 2, 5], dtype=torch.int32) if packed else None
    lead, seqs = ((5,), 3) if packed else ((2, 3), 2)
    x, w, b, s = (_randn(gen, *lead, 2), _randn(gen, 2, 3), _randn(gen, 2), _randn(gen, seqs, 2, 2))
    assert torch.autograd.gradcheck(lambda *a: ref.conv(a[0], a[1], a[2], True, a[3], off),
                                    (x, w, b, s))
    u, dt, g = (_randn(gen, *lead, 2) for _ in range(3))
    B, C = (_randn(gen, *lead, 1, 3) for _ in range(2))
    A, skip, bias, h = _randn(gen, 2, 3), _randn(gen, 2), _randn(gen, 2), _randn(gen, seqs, 2, 3)
    assert torch.autograd.gradcheck(
        lambda *a: ref.scan(*a[:8], True, a[8], off), (u, dt, A, B, C, skip, g, bias, h))


def test_reference_scan_is_a_convolution_when_nothing_varies():
    """With constant d, B and C the scan is the causal convolution with the
    kernel K_t = sum_n C[n] exp(d A[n] t) d B[n]."""
    gen = torch.Generator().manual_seed(1)
    T, n, d = 20, 4, 0.3
    u = torch.randn(1, T, 1, generator=gen, dtype=torch.float64)
    A = -torch.rand(1, n, generator=gen, dtype=torch.float64) * 3
    B, C = (torch.randn(n, generator=gen, dtype=torch.float64) for _ in range(2))
    y, _ = ref.scan(u, torch.full_like(u, d), A, B.expand(1, T, 1, n), C.expand(1, T, 1, n))
    t = torch.arange(T, dtype=torch.float64)
    K = (C * torch.exp(d * A * t[:, None]) * d * B).sum(-1)
    want = [sum(K[j] * u[0, i - j, 0] for j in range(i + 1)) for i in range(T)]
    assert torch.allclose(y[0, :, 0], torch.stack(want), rtol=1e-12, atol=1e-12)


def test_reference_conv_by_hand():
    x = torch.tensor([1.0, 2.0, 3.0], dtype=torch.float64).reshape(1, 3, 1)
    w = torch.tensor([[10.0, 1.0]], dtype=torch.float64)
    y, last = ref.conv(x, w, state=torch.tensor([[[5.0]]], dtype=torch.float64))
    assert y.flatten().tolist() == [51.0, 12.0, 23.0] and last.item() == 3.0


def test_token_scan_of_too_many_entries(seq):
    """Entries are counted in 32 bits, in steps of up to four for each of 65535
    blocks: beyond 2^31 - 1 - 4 * 65535 a step past the last one would wrap."""
    for n in (2 ** 31 - 4 * 65535, 2 ** 31 - 1):
        a = scan_args(seq, rows=1, sequences=n, slots=0x10000, num_slots=1)
        assert seq._lib().tcu_state_scan_step(a, None) == UNSUPPORTED


def test_pitches_beyond_32_bits_are_refused(seq):
    far = seq._Rows(0x10000, 2 ** 33, 2 ** 31)
    for k in ("x", "y", "dy", "dx"):
        assert seq._lib().tcu_short_conv(conv_args(seq, **{k: far}), None) == UNSUPPORTED
    for k in ("u", "dt", "gate", "y", "B", "C", "dB"):
        assert seq._lib().tcu_state_scan(scan_args(seq, **{k: far}), None) == UNSUPPORTED
    for k in ("u", "dt", "gate", "y", "B", "C"):
        a = scan_args(seq, rows=1, slots=0x10000, num_slots=1, **{k: far})
        assert seq._lib().tcu_state_scan_step(a, None) == UNSUPPORTED
