"""The paged rollouts example: all paged-cache entry points as one layer, against
the same layer on the ring cache."""

import importlib.util
import os

import pytest
import torch

from paper_2605_30351_gb300 import videomla as V

pytestmark = pytest.mark.gpu
PATH = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples",
                    "paged_rollouts.py")


def test_rollouts_match_the_ring_cache():
    """Both sides round keys, weights and outputs to bf16 at the same places, but
    not the rotated queries: 2^-9 of a score's positional part (of size about 1)
    there, and bf16 outputs on either side: 1e-2 in relative 2-norm."""
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    spec = importlib.util.spec_from_file_location("paged_rollouts", PATH)
    ex = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(ex)
    V.mla_device_status(clear=True)
    worst, used, layer = ex.main()
    assert worst <= 1e-2
    # rollout 1: 4 frames, shares 2 of them with its branch 3; rollout 2: 5 frames.
    # Frames of 64 tokens fill 4 pages of 16: 4 + (4 - 2) + 5 frames
    T = layer.T
    assert layer.lens == [0, 4 * T, 5 * T, 4 * T]
    assert used == (4 + 2 + 5) * 4
    n = int((layer.cache.refs > 0).sum())
    assert layer.cache.lens.tolist() == layer.lens and n == used
