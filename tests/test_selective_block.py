"""The example of the sequence operators: what it prints, held to bounds set
before its first run."""
import importlib.util
import os

import pytest

pytestmark = pytest.mark.gpu
HERE = os.path.dirname(os.path.abspath(__file__))


@pytest.fixture(scope="module")
def example():
    from paper_1908_06649_gb300 import _build
    _build.build()
    path = os.path.join(os.path.dirname(HERE), "examples", "selective_block.py")
    spec = importlib.util.spec_from_file_location("selective_block", path)
    m = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(m)
    return m


def test_tokens_continue_packed_prompts(example):
    """bf16 throughout: four roundings of 2^-8 on the way to an output."""
    assert example.serve(example.Block()) <= 4 * 2.0 ** -8


def test_a_block_learns(example):
    first, last = example.train(example.Block())
    assert last < first


def test_invariant_scan_is_the_dft_convolution(example):
    """fp32 scan of 2048 rows, decays of at most 1e-1 a row (so some hundred
    rows in memory), and a 3xTF32 convolution held to 1e-5 of its inputs."""
    assert example.invariant() <= 5e-5
