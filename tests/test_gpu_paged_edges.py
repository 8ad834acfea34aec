"""Attention over the paged latent cache where its inputs lie at an edge of what the
entry point accepts."""

import pytest
import torch

from paper_2605_30351_gb300 import videomla as V
from test_gpu_paged_attention import Problem

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    V.load()
    V.mla_device_status(clear=True)
    yield
    assert V.mla_device_status(clear=True) == V.MLA_OK


@pytest.mark.parametrize("d_c,d_r", [(64, 32), (128, 64), (192, 32), (256, 64), (512, 64)])
@pytest.mark.parametrize("lens,new,heads", [
    ([9000], [1], 12),                  # one tile of 16 rows, cut by many shares
    ([9000, 300], [2, 2], 12),          # short tiles: partial rows row after row
    ([9000], [10], 12),                 # a whole tile cut by many shares
    ([600] * 60, [9] * 60, 12),         # tiles cut by two or three shares
])
def test_workspace_at_any_16_byte_boundary(d_c, d_r, lens, new, heads):
    """A workspace of the size asked for, inside a larger buffer at each 16-byte
    offset of 64 bytes: the same bits, and the bytes around it as they were."""
    p = Problem(lens, new, d_c=d_c, d_r=d_r, heads=heads, page=32, seed=d_c)
    ref = p.run(1)
    p.check(ref, 1, tokens=2)
    need = p.workspace.numel()
    arena = torch.empty(need + 192, dtype=torch.uint8, device="cuda")
    assert arena.data_ptr() % 64 == 0
    for off in (64, 80, 96, 112):
        arena.fill_(0xA5)
        p.workspace = arena[off:off + need]
        assert torch.equal(p.run(1), ref), off
        assert (arena[:off] == 0xA5).all() and (arena[off + need:] == 0xA5).all(), off
