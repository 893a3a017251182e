"""The waits of the attention kernels and the recurrence, read in their sources: none is cut short
on a GPU to see what follows.

A wait ends after two seconds.  Where it runs out for some threads and not for
others, a thread that leaves a loop while others go on to a barrier of a fixed
count would leave them there for ever; so a warp has one verdict, and threads
that share a barrier stay in their loops."""
import os
import re

import pytest

from paper_1908_06649_gb300 import _build

FILES = ["window_attention.cu", "window_attention_grad.cu", "window_attention_step.cu"]


def source(name):
    with open(os.path.join(_build.CSRC, name)) as f:
        return re.sub(r"//[^\n]*", "", f.read())


@pytest.mark.parametrize("name", FILES)
def test_waits_have_one_verdict_a_warp(name):
    text = source(name)
    assert not re.search(r"\bmbar_(try_)?wait", text)
    assert "while (true)" not in text
    body = re.search(r"bool warp_waits\([^{]*\{(.*?)\n\}", source("attn_common.cuh"), re.S).group(1)
    assert "__all_sync(~0u, mbar_wait_bounded(" in body


def test_waits_of_the_recurrence_have_one_verdict_a_warp():
    text = source("gated_scan.cu")
    waits = re.findall(r"[^\n]*\bmbar_(?:try_)?wait\w*\([^\n]*", text)
    assert len(waits) == 1 and "__all_sync(~0u, mbar_wait_cluster_bounded(" in waits[0]


def test_no_thread_leaves_others_at_a_barrier():
    """A barrier of a fixed count lies in no branch out of which a thread of
    its group can go early."""
    kernels = re.split(r"\n__global__ ", re.sub(r"template <[^>]*>", "", source("window_attention_grad.cu")))
    with_barriers = [k for k in kernels if re.search(r"\bbar\.sync", k)]
    assert len(with_barriers) == 2
    for k in with_barriers:
        k = k[:k.index("\n}\n")]
        for at in (m.start() for m in re.finditer(r"\bbar\.sync", k)):
            # the innermost role of warps around the barrier: from `} else {` at the
            # kernel's own indentation to the block's end
            lo = max(k.rfind("\n  } else", 0, at), k.rfind("\n  if (warp", 0, at))
            hi = k.index("\n  }", at)
            role = k[lo:hi]
            assert not re.search(r"\b(break|return|goto|continue)\b", role), role
            assert not re.search(r"for \([^;]*;[^;]*\bok\b", role), role
