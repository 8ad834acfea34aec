"""The sliding-rollouts example runs, its pool stays small, and its layer agrees with the
framework's sink ring: both are within 1e-2 (relative norm) of the float64 layer, the bound of
the ring's own tests, so within 2e-2 of each other."""

import importlib.util
import os

import pytest
import torch

pytestmark = pytest.mark.gpu

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def test_example():
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    spec = importlib.util.spec_from_file_location(
        "sliding_rollouts", os.path.join(ROOT, "examples", "sliding_rollouts.py"))
    m = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(m)
    worst, held, gone = m.main(chunks=12, rollouts=2, frames=2)
    assert worst <= 2e-2
    assert [h + g for h, g in zip(held, gone)] == [12 * 128] * 2
    assert max(held) <= 64 + 16 + 256                # sink, the page before the kept, kept
