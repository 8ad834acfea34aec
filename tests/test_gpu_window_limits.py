"""Where the streams of a sliding window end: lists cut back into the sinks' pages."""

import numpy as np
import pytest
import torch

from oracle import paged_oracle as O
from paper_2605_30351_gb300 import videomla as V

pytestmark = pytest.mark.gpu

I32, BF16 = torch.int32, torch.bfloat16


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    V.load()
    V.mla_device_status(clear=True)
    yield
    assert V.mla_device_status(clear=True) == V.MLA_OK


def i32(v):
    return torch.tensor(np.asarray(v), dtype=I32, device="cuda")


def ints(*shape):
    return torch.full(shape, -9, dtype=I32, device="cuda")


@pytest.mark.parametrize("cut,new", [(90, 28), (90, 5), (111, 1), (111, 3), (112, 1), (112, 40), (1, 200)])
def test_a_list_cut_back_into_the_sinks_pages(cut, new):
    """100 sinks in pages of 16 take 112 places. A stream that gave tokens back and is cut to
    fewer has no index for what it grows by: positions refuses that step as attention does,
    and no other stream's. The second stream gave nothing back: its sinks may grow."""
    page, sinks, window = 16, 100, 50
    cache = V.PagedCache.empty(1, 60, page, 2, 30, 64, 32)
    win = V.PagedWindow(window, sinks, i32([0, 0]))
    V.mla_pages_resize(cache, i32([240, 60]))
    V.mla_pages_slide(cache, win, i32([60, -1]))
    back = win.dropped.tolist()
    assert back == [64, 0]
    V.mla_pages_resize(cache, i32([cut, -1]))
    n = i32([new, 30])
    q_start, lens, total = ints(3), ints(2), new + 30
    V.mla_paged_window_plan(cache, win, n, q_start, lens)
    V.mla_pages_resize(cache, lens)
    assert cache.lens.tolist() == [cut + new, 90] and V.mla_device_status(clear=True) == V.MLA_OK
    pos, beside, rows = ints(total, 3), ints(total, 3), ints(total)
    V.mla_paged_window_positions(cache, win, q_start, 1, 8, 4, pos, beside, rows)
    refused = cut < 112
    assert V.mla_device_status(clear=True) == (V.MLA_ERR_RANGE if refused else V.MLA_OK)
    want, apart, at = [], [], []
    for s, (k, b, m) in enumerate(zip(cache.lens.tolist(), back, n.tolist())):
        x, y = O.window_positions(k, b, m, 1, window, sinks, 8, 4, page)
        want += x
        apart += y
        table = cache.table[s].tolist()
        at += [-1 if s == 0 and refused else table[p // page] * page + p % page for p in range(k - m, k)]
    if refused:
        assert want[:new] == apart[:new] == [(0, 0, 0)] * new
    else:                                             # the place behind the sinks' pages, and 64
        assert want[0] == (176 // 8, 0, 0)
    assert pos.tolist() == [list(v) for v in want]
    assert beside.tolist() == [list(v) for v in apart]
    assert rows.tolist() == at
    q = torch.zeros(total, 1, 64, dtype=BF16, device="cuda")
    o = torch.full_like(q, 7.0)
    ws = torch.empty(V.mla_paged_workspace_bytes(cache), dtype=torch.uint8, device="cuda")
    V.mla_paged_window_attention(cache, win, 0, q, q[:, :, :32].contiguous(), None, q_start, 128, 1, ws, o)
    assert V.mla_device_status(clear=True) == (V.MLA_ERR_RANGE if refused else V.MLA_OK)
    assert (o[:new] == (7.0 if refused else 0.0)).all() and (o[new:] == 0).all()
