"""Where the streams of a sliding window end: lists cut back into the sinks' pages, the rotary
table, windows shorter than a block."""

import importlib.util
import os

import numpy as np
import pytest
import torch

from oracle import paged_oracle as O
from paper_2605_30351_gb300 import videomla as V

pytestmark = pytest.mark.gpu

I32, BF16 = torch.int32, torch.bfloat16
ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
# weights and output are rounded to bf16 once each; scores move a weight by less than 2^-10
REL = 2 * 2.0 ** -8 + 2.0 ** -10


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


def test_a_stream_past_the_usual_table():
    """Coordinates are absolute, so a stream goes as far as its rotary table: the 1,024
    positions that a configuration has by default, or as many as the caller makes. Tokens 1,000 to
    1,047 of a stream: with the longer table their keys and queries are those of the formula's
    angles; with the short one each coordinate past its end is recorded, by the append and by the
    rotation, and counts as 0."""
    page, new, m = 16, 48, 16
    cache = V.PagedCache.empty(1, 8, page, 1, 7, 64, 32)
    win = V.PagedWindow(30, 4, i32([0]))
    V.mla_pages_resize(cache, i32([40]))
    win.dropped.fill_(960)
    q_start, lens, pos, rows = ints(2), ints(1), ints(new, 1), ints(new)
    V.mla_paged_window_plan(cache, win, i32([new]), q_start, lens)
    V.mla_pages_resize(cache, lens)
    V.mla_paged_window_positions(cache, win, q_start, 1, 1, 1, pos, None, rows)
    assert pos[:, 0].tolist() == list(range(1000, 1048)) and V.mla_device_status(clear=True) == V.MLA_OK
    g = torch.Generator(device="cuda").manual_seed(3)
    c, kr, q = (torch.randn(new, *s, device="cuda", generator=g).to(BF16) for s in ((64,), (32,), (3, 32)))
    freq = 10000.0 ** (-np.arange(m) / m)
    for length in (1048, 1024, 4096):
        rope = V.Rope(torch.from_numpy(V.mla_rope_scaled_table_fill(32, length)).cuda(), (m, 0, 0), axes=1)
        inside = np.array([p < length for p in range(1000, 1048)])
        y = torch.empty_like(q)
        for call in (lambda: V.mla_paged_append(cache, 0, c, kr, q_start, pos, rope),
                     lambda: V.mla_rope_apply(rope, q, pos, y)):
            call()
            assert V.mla_device_status(clear=True) == (V.MLA_OK if inside.all() else V.MLA_ERR_RANGE), length
        angle = np.where(inside, np.arange(1000, 1048), 0)[:, None] * freq
        cos, sin = np.cos(angle), np.sin(angle)
        got = cache.kr[0].view(-1, 32)[rows.long()]
        for x, z in ((kr[:, None], got[:, None]), (q, y)):
            x, z = x.double().cpu().numpy(), z.double().cpu().numpy()
            a, b = x[..., ::2], x[..., 1::2]
            # one rounding to bf16; the table's (2^-24) and three of fp32 arithmetic on |a|, |b|
            for ref, out in ((a * cos[:, None] - b * sin[:, None], z[..., ::2]),
                             (a * sin[:, None] + b * cos[:, None], z[..., 1::2])):
                bound = 2.0 ** -8 * np.abs(ref) + 2.0 ** -21 * (np.abs(a) + np.abs(b))
                assert (np.abs(out - ref) <= bound).all(), length


def test_a_stream_shifted_back_by_a_constant():
    """Scores depend on distances only: a stream across the end of the usual table gives what
    the same stream gives 1,000 positions earlier. A rotated key or query is off by a rounding of 2^-8
    of its size, so a score by (2 * 2^-8 + 2^-16) sum |q_r| |k| / sqrt(128) in each of the two, sums over
    the pairs; weights by a factor of exp of twice that; on top of the two rounding bounds."""
    page, new, d_r = 16, 40, 32
    rope = V.Rope(torch.from_numpy(V.mla_rope_scaled_table_fill(d_r, 2048)).cuda(), (16, 0, 0), axes=1)
    g = torch.Generator(device="cuda").manual_seed(8)
    held = 100
    c, kr = (torch.randn(held, w, device="cuda", generator=g).to(BF16) for w in (64, d_r))
    q_c, q_r = (torch.randn(new, 4, w, device="cuda", generator=g).to(BF16) for w in (64, d_r))
    outs, keys = [], []
    for first in (0, 960):                            # tokens given back: whole pages
        cache = V.PagedCache.empty(1, 8, page, 1, 8, 64, d_r)
        win = V.PagedWindow(50, 0, i32([0]))
        V.mla_pages_resize(cache, i32([held]))
        win.dropped.fill_(first)
        pos, q = ints(held, 1), torch.empty_like(q_r)
        start = i32([0, held])
        V.mla_paged_window_positions(cache, win, start, 1, 1, 1, pos)
        V.mla_paged_append(cache, 0, c, kr, start, pos, rope)
        V.mla_rope_apply(rope, q_r, pos[-new:].contiguous(), q)
        o, ws = torch.empty_like(q_c), torch.empty(V.mla_paged_workspace_bytes(cache), dtype=torch.uint8, device="cuda")
        V.mla_paged_window_attention(cache, win, 0, q_c, q, None, i32([0, new]), 128, 1, ws, o)
        outs.append(o.double().cpu().numpy())
    assert pos[-1, 0] == 1059 and V.mla_device_status(clear=True) == V.MLA_OK
    kd, qd = kr.double().cpu().numpy(), q_r.double().cpu().numpy()
    norm = lambda x: np.hypot(x[..., ::2], x[..., 1::2])  # noqa: E731  turned channels are within it
    for i in range(new):
        p = held - new + i
        sees = range(max(0, p - 49), p + 1)
        v = np.abs(c.double().cpu().numpy()[list(sees)])
        worst = max((norm(qd[i]) @ norm(kd[j])).max() for j in sees)
        shift = 2 * (2 * 2.0 ** -8 + 2.0 ** -16) * worst / 128 ** 0.5
        bound = (np.exp(2 * shift) - 1 + 2 * REL) * v.max(0)
        assert (np.abs(outs[0][i] - outs[1][i]) <= bound).all(), i


def test_the_example_past_the_usual_table():
    """1,032 frames: more than the 1,024 positions of a default table. Its layer agrees with
    the sink ring, which numbers held frames anew for every window; both are within 1e-2 (relative
    norm) of the float64 layer, the bound of the ring's own tests, so within 2e-2 of each other."""
    spec = importlib.util.spec_from_file_location(
        "sliding_rollouts", os.path.join(ROOT, "examples", "sliding_rollouts.py"))
    m = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(m)
    worst, held, gone = m.main(chunks=172, rollouts=1, frames=6)
    assert worst <= 2e-2
    assert [h + g for h, g in zip(held, gone)] == [1032 * 64]


@pytest.mark.parametrize("window,block", [(20, 32), (1, 8), (31, 32), (32, 32), (50, 100)])
def test_a_window_shorter_than_a_block(window, block):
    """Blocks longer than the window: the next block sees no key of those before it, so
    max(0, window - block) tokens are kept. The list stays short however long the stream gets,
    and a block's rows see the newest keys of their own block and the sinks."""
    page, sinks = 16, 5
    most = -(-sinks // page) + -(-(max(0, window - block) + page + block) // page)
    cache = V.PagedCache.empty(1, most + 1, page, 1, most, 64, 32)
    win = V.PagedWindow(window, sinks, i32([0]))
    keep, n = i32([max(0, window - block)]), i32([block])
    q_start, lens = ints(2), ints(1)
    g = torch.Generator(device="cuda").manual_seed(window)
    ws = torch.empty(V.mla_paged_workspace_bytes(cache), dtype=torch.uint8, device="cuda")
    rope = V.Rope(torch.from_numpy(V.mla_rope_scaled_table_fill(32, 40 * block)).cuda(), (16, 0, 0), axes=1)
    pos = ints(block, 1)
    for step in range(40):
        V.mla_paged_window_plan(cache, win, n, q_start, lens)
        V.mla_pages_resize(cache, lens)
        V.mla_paged_window_positions(cache, win, q_start, block, 1, 1, pos)
        assert pos[:, 0].tolist() == list(range(step * block, (step + 1) * block))
        c, kr, q_c, q_r = (torch.randn(*s, device="cuda", generator=g).to(BF16) for s in
                           ((block, 64), (block, 32), (block, 4, 64), (block, 4, 32)))
        V.mla_paged_append(cache, 0, c, kr, q_start, pos, rope)
        o = torch.full_like(q_c, float("nan"))
        V.mla_paged_window_attention(cache, win, 0, q_c, q_r, None, q_start, 128, block, ws, o)
        if step in (0, 1, 7, 39):
            held, gone = int(cache.lens[0]), int(win.dropped[0])
            a = np.arange(held)
            ids = cache.table[0].cpu().numpy()[a // page]
            k, r = (t[0].double().cpu().numpy()[ids, a % page] for t in (cache.c, cache.kr))
            sees = O.window_sees(held - 1, held, gone, block, window, sinks, page)
            for i in (0, block - 1):                  # the rows of a block see the same
                ref, size = O.attend_window(q_c[i].double().cpu().numpy(), *2 * [q_r[i].double().cpu().numpy()],
                                            k, r, sees, 128)
                assert (np.abs(o[i].double().cpu().numpy() - ref) <= REL * size).all(), (step, i)
        V.mla_pages_slide(cache, win, keep)
    assert V.mla_device_status(clear=True) == V.MLA_OK
    assert int(cache.lens[0] + win.dropped[0]) == 40 * block


def test_a_negative_count_to_keep():
    """-1 leaves a stream alone; any other negative count, as w - b of a block longer than the
    window, is recorded too."""
    cache = V.PagedCache.empty(1, 40, 8, 3, 12, 8, 8)
    win = V.PagedWindow(5, 3, i32([0, 0, 0]))
    V.mla_pages_resize(cache, i32([60, 60, 60]))
    for bad in (-2, -12, -2 ** 31):
        V.mla_pages_slide(cache, win, i32([-1, bad, -1]))
        assert V.mla_device_status(clear=True) == V.MLA_ERR_RANGE, bad
        assert cache.lens.tolist() == [60] * 3 and win.dropped.tolist() == [0] * 3
    V.mla_pages_slide(cache, win, i32([-1, -7, 20]))
    assert V.mla_device_status(clear=True) == V.MLA_ERR_RANGE
    assert cache.lens.tolist() == [60, 60, 28] and win.dropped.tolist() == [0, 0, 32]
    V.mla_pages_slide(cache, win, i32([-1, -1, -1]))
    assert V.mla_device_status(clear=True) == V.MLA_OK


def test_coordinates_beside_the_sinks_in_long_blocks():
    """In blocks of at most window + sinks tokens no coordinate beside the sinks is negative; in
    longer ones it is for tokens far before their window, and the rotation records it."""
    page, window, sinks = 16, 20, 12
    rope = V.Rope(torch.from_numpy(V.mla_rope_scaled_table_fill(32, 512)).cuda(), (16, 0, 0), axes=1)
    for block in (7, 32, 33, 100, 0):
        cache = V.PagedCache.empty(1, 30, page, 1, 30, 8, 8)
        V.mla_pages_resize(cache, i32([300]))
        win, pos, beside = V.PagedWindow(window, sinks, i32([0])), ints(300, 1), ints(300, 1)
        V.mla_paged_window_positions(cache, win, i32([0, 300]), block, 1, 1, pos, beside)
        assert V.mla_device_status(clear=True) == V.MLA_OK
        want, apart = O.window_positions(300, 0, 300, block, window, sinks, 1, 1, page)
        assert pos[:, 0].tolist() == [v[0] for v in want]
        assert beside[:, 0].tolist() == [v[0] for v in apart]
        low = int(beside.min())
        assert (low < 0) == (block in (33, 100, 0)), (block, low)
        x = torch.randn(300, 1, 32, device="cuda").to(BF16)
        V.mla_rope_apply(rope, x, beside, torch.empty_like(x))
        assert V.mla_device_status(clear=True) == (V.MLA_ERR_RANGE if low < 0 else V.MLA_OK)


@pytest.mark.parametrize("window,block,page", [(16, 16, 16), (20, 32, 8), (1, 8, 8), (30, 48, 24)])
def test_a_stream_without_sinks_keeps_its_count(window, block, page):
    """A window of no more than the next block keeps nothing of what is held. Without sinks and with
    whole pages all of it could go; but a stream that holds no token starts anew, at index 0, so a slide
    leaves the last page. A stream that ended does start anew."""
    cache = V.PagedCache.empty(1, 24, page, 2, 12, 8, 8)
    win = V.PagedWindow(window, 0, i32([0, 0]))
    n, keep = i32([block, block]), i32([max(0, window - block)] * 2)
    q_start, lens, pos = ints(3), ints(2), ints(2 * block, 1)
    first = [0, 0]
    for step in range(30):
        V.mla_paged_window_plan(cache, win, n, q_start, lens)
        V.mla_pages_resize(cache, lens)
        V.mla_paged_window_positions(cache, win, q_start, block, 1, 1, pos)
        assert pos[:, 0].tolist() == [f + i for f in first for i in range(block)], step
        V.mla_pages_slide(cache, win, keep)
        assert all(0 < k <= page for k in cache.lens.tolist())
        first = [f + block for f in first]
        if step == 11:
            V.mla_pages_resize(cache, i32([-1, 0]))
            first[1] = 0
    assert V.mla_device_status(clear=True) == V.MLA_OK
