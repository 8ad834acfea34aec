"""Page copies whose piece counts pass 31 bits."""

import pytest
import torch

from paper_2605_30351_gb300 import videomla as V

pytestmark = pytest.mark.gpu


def test_pages_of_two_to_the_31_pieces():
    """Pages of 2^18 rows of 65,536 values: 2^31 pieces of 16 bytes, 32 GiB each. A copy
    of a page, then a branch that grows: its own copy of all rows but the last one."""
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    rows, width, pages = 1 << 18, 1 << 16, 2
    if torch.cuda.mem_get_info()[0] < (80 << 30):
        pytest.skip("64 GiB of the GPU's memory are not free")
    V.load()
    V.mla_device_status(clear=True)
    cache = V.PagedCache.empty(1, pages, rows, 2, 1, width, 8)
    g = torch.Generator().manual_seed(1)
    at = torch.cat((torch.tensor([0, 1, rows // 2 - 1, rows // 2, rows - 2, rows - 1]),
                    torch.randint(0, rows, (200,), generator=g))).unique().cuda()
    c = torch.randn(at.numel(), width, generator=g).to(torch.bfloat16).cuda()
    kr = torch.randn(at.numel(), 8, generator=g).to(torch.bfloat16).cuda()
    cache.c[0, 0, at], cache.kr[0, 0, at] = c, kr

    def ints(v):
        return torch.tensor(v, dtype=torch.int32, device="cuda")

    V.mla_pages_copy(cache, ints([0]), ints([1]))
    for page in (0, 1):
        assert torch.equal(cache.c[0, page, at], c) and torch.equal(cache.kr[0, page, at], kr)
    cache.c[0, 1].zero_()
    cache.kr[0, 1].zero_()
    cache.table.copy_(ints([[0], [0]]))
    cache.lens.copy_(ints([rows - 1, rows - 1]))
    cache.refs.copy_(ints([2, 0]))
    V.mla_pages_resize(cache, ints([-1, rows]))
    held = at < rows - 1
    assert cache.table.tolist() == [[0], [1]] and cache.refs.tolist() == [1, 1]
    assert cache.lens.tolist() == [rows - 1, rows]
    assert torch.equal(cache.c[0, 1, at[held]], c[held])
    assert torch.equal(cache.kr[0, 1, at[held]], kr[held])
    assert (cache.c[0, 1, rows - 1] == 0).all() and (cache.c[0, 0, at] == c).all()
    assert V.mla_device_status(clear=True) == V.MLA_OK
