"""Every form of attention over a sliding window, at every size: the library chooses among teams
of 1 to 8 CTAs, shares of 16-row tiles, and tiles of 128 and 256 rows by estimated times, so that the
form that a call of the other tests takes may change with the estimates. Here each is named. The
bound of a value is that of test_gpu_paged_window."""

import numpy as np
import pytest
import torch

import test_gpu_paged_window as T
from oracle import paged_oracle as O
from paper_2605_30351_gb300 import videomla as V

pytestmark = pytest.mark.gpu

TEAMS, SHARES, TILES, PAIRS = (1, 2, 4, 8), 16, 128, 256
FORMS = (*TEAMS, SHARES, TILES, PAIRS)
WIDTHS = [(d_c, d_r) for d_c in (64, 128, 192, 256) for d_r in (32, 64)]
# every instance of every kernel; at d_c = 512 there is one form
INSTANCES = [(*w, f) for w in WIDTHS for f in FORMS] + [(512, 32, TILES), (512, 64, TILES)]


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    V.load()
    V.mla_device_status(clear=True)
    yield
    assert V.mla_device_status(clear=True) == V.MLA_OK


@pytest.fixture(autouse=True)
def _restore():
    yield
    V.mla_selftest_window_form(0)


def run(form, p, tokens=None):
    """The call in this form, held against the oracle; nothing was recorded."""
    V.mla_selftest_window_form(form)
    o = T.run_check(p, tokens)
    assert V.mla_selftest_window_form(0) == form
    assert V.mla_device_status(clear=True) == V.MLA_OK
    return o


@pytest.mark.parametrize("d_c,d_r,form", INSTANCES)
def test_shapes(d_c, d_r, form):
    """One token, an idle stream, pages that end inside a key tile or span several, more rows than
    a row tile, streams shorter and longer than window and sinks; sinks that end off 16
    tokens and off pages, with queries of their own or without."""
    for page, sinks in ((8, 21), (16, 21), (64, 70), (100, 130)):
        for turned in (True, False):
            run(form, T.Problem([1, 300, 77, 530, 129], [1, 30, 0, 5, 129], 90, sinks, gone=[0, page, 0, page * 2, 0],
                                heads=12, d_c=d_c, d_r=d_r, page=page, turned=turned, seed=d_c + page), 5)


@pytest.mark.parametrize("form", FORMS)
@pytest.mark.parametrize("sinks", [0, 1, 64, 100, 130, 1 << 30])
def test_window_edges(form, sinks):
    """Windows and sinks that end inside tiles, meet, overlap, or are longer than the stream."""
    for window in (1, 2, 16, 17, 64, 127, 128, 129, 1000, 1 << 30):
        for new, d_c in (([1, 1, 2], 64), ([90, 9, 33], 128)):
            run(form, T.Problem([400, 9, 131], new, window, sinks, d_c=d_c, seed=window % 97 + sinks % 89,
                                turned=window % 2 == 0), 6)


@pytest.mark.parametrize("form", FORMS)
@pytest.mark.parametrize("d_c", [64, 192])
def test_blocks(form, d_c):
    """No mask, token by token, blocks that end inside tiles and before the newest token's block
    does, longer and shorter than the window (keys between the windows of a tile's blocks hold NaN);
    blocks count from a stream's start, given back or not."""
    for block in (0, 1, 2, 7, 64, 100, 1 << 30):
        for window in (20, 77):
            for gone in (None, [48, 0, 160, 0]):
                run(form, T.Problem([333, 200, 150, 1], [150, 200, 64, 1], window, 30, block, gone=gone, d_c=d_c,
                                    turned=window == 20), 6)
                run(form, T.Problem([333, 200, 150, 1], [3, 1, 2, 1], window, 30, block, gone=gone, d_c=d_c), 6)


@pytest.mark.parametrize("d_c,d_r", WIDTHS)
def test_blocks_in_pairs(d_c, d_r):
    """Tiles of 256 rows mask hidden keys in two ways, token by token and by blocks of the mask."""
    for block, window, page in ((0, 40, 16), (7, 100, 64), (64, 300, 100), (100, 20, 32), (1, 130, 24)):
        for sinks in (0, 70):
            run(PAIRS, T.Problem([600, 200, 150, 1], [300, 200, 64, 1], window, sinks, block, heads=12, d_c=d_c,
                                 d_r=d_r, page=page, turned=block != 7, gone=[page * 2, 0, 0, 0]), 6)


@pytest.mark.parametrize("form", FORMS)
@pytest.mark.parametrize("page", [8, 24, 32, 48, 96, 120, 128, 200, 256])
def test_page_sizes(form, page):
    for new, d_c in ((2, 256), (40, 128)):
        for turned in (True, False):
            run(form, T.Problem([700, 3, 1700], [new, 2, new], 300, 130, gone=[page * 2, 0, page * 3], page=page,
                                heads=5, d_c=d_c, turned=turned), 5)


@pytest.mark.parametrize("form", FORMS)
def test_odd_page_sizes(form):
    """Pages of any size from 8 tokens on, odd ones and longer than several blocks of keys."""
    for page in (9, 13, 50, 127, 129, 300):
        front = O.front(70, page)
        for turned in (True, False):
            run(form, T.Problem([front + 450, 3, 700], [40, 2, 1], 150, 70, gone=[page * 2, 0, 0], page=page, heads=5,
                                d_c=128, turned=turned), 5)
            if form == TILES:
                run(form, T.Problem([front + 450, 3, 700], [40, 2, 1], 150, 70, gone=[page * 2, 0, 0], page=page,
                                    heads=5, d_c=512, turned=turned), 5)


@pytest.mark.parametrize("form", FORMS)
def test_as_many_slots_as_there_may_be(form):
    """65,536 slots, six of them with work."""
    seqs = 65536
    lens, new = [0] * seqs, [0] * seqs
    for s, (k, n) in zip((0, 1, 777, 40000, 65534, 65535), ((300, 1), (40, 30), (90, 2), (5, 5), (400, 1), (33, 4))):
        lens[s], new[s] = k, n
    run(form, T.Problem(lens, new, 64, 10, heads=3, d_c=128), 4)


@pytest.mark.parametrize("page", [8, 24, 48, 64, 100, 200])
def test_page_sizes_of_the_widest(page):
    for new in (1, 5, 40):
        for turned in (True, False):
            run(TILES, T.Problem([700, 3, 1700], [new, 2, new], 300, 130, gone=[0, 0, page * 3], page=page, heads=5,
                                 d_c=512, d_r=64, turned=turned), 5)


@pytest.mark.parametrize("form", FORMS)
def test_head_counts(form):
    for heads in (1, 3, 16, 40, 200):
        for new in (1, 17):
            run(form, T.Problem([260, 40], [new, new], 100, 12, heads=heads, d_c=128), 4)


@pytest.mark.parametrize("form", FORMS)
def test_rows_that_see_nothing(form):
    """More new tokens than the stream holds; empty streams."""
    run(form, T.Problem([3, 0, 130, 0], [9, 4, 140, 0], 20, 2, heads=12))
    run(form, T.Problem([0, 0], [1, 2], 20, 2, block=0))
    run(form, T.Problem([0], [1], 20, 0))
    run(form, T.Problem([4], [300], 2, 0, block=3, d_c=192))


@pytest.mark.parametrize("form", FORMS)
def test_long_streams(form):
    """Work split along the keys and joined, or walked by one CTA; the same bits each time."""
    for lens, new, window, sinks, page in (([9001, 70, 1, 12011], [1, 70, 1, 30], 4096, 200, 64),
                                           ([3000] * 7, [1] * 7, 1500, 4, 48)):
        p = T.Problem(lens, new, window, sinks, heads=12, d_c=192, page=page, seed=9)
        o = run(form, p, 4)
        V.mla_selftest_window_form(form)
        p.workspace.fill_(255)
        assert torch.equal(o, p.run())


@pytest.mark.parametrize("form", FORMS)
def test_many_streams(form):
    seqs = 300
    lens = [(37 * s) % 300 + 10 for s in range(seqs)]
    new = [3 if s % 5 == 0 else 0 for s in range(seqs)]
    new[7] = lens[7] = 90
    run(form, T.Problem(lens, new, 100, 10, gone=[16 * (s % 4) if lens[s] - new[s] > 20 else 0 for s in range(seqs)],
                        heads=12), 3)


@pytest.mark.parametrize("form", FORMS)
def test_random_calls(form):
    """Sizes and masks drawn at random, keys that no row sees NaN or infinite."""
    rng = np.random.default_rng(form)
    for k in range(60):
        seqs = int(rng.integers(1, 6))
        page = int(rng.choice([8, 16, 24, 64, 100, 128]))
        sinks = int(rng.choice([0, 1, 5, 60, 200]))
        wide = rng.random() < 0.6
        new = [int(rng.integers(0, 60 if wide else 3)) for _ in range(seqs)]
        if sum(new) == 0:
            new[0] = 1
        gone = [int(rng.integers(0, 9)) * page for _ in range(seqs)]
        front = O.front(sinks, page)
        lens = [int(rng.integers(n + (front if g else 0), n + front + 500)) for n, g in zip(new, gone)]
        d_c, d_r = WIDTHS[int(rng.integers(len(WIDTHS)))]
        if form == TILES and rng.random() < 0.3:
            d_c = 512
        run(form, T.Problem(lens, new, int(rng.integers(1, 400)), sinks, block=int(rng.choice([0, 1, 1, 3, 50, 130])),
                            gone=gone, turned=bool(rng.random() < 0.6), heads=int(rng.choice([1, 4, 12])), d_c=d_c,
                            d_r=d_r, page=page, seed=k), 5)


@pytest.mark.parametrize("form", FORMS)
def test_what_a_row_sees_reaches_it(form):
    """A NaN in a sink or window key that rows see reaches them, wherever the work is cut."""
    for new in (1, 40):
        for where in (2, 5990):
            p = T.Problem([6000], [new], 3000, 16, dirty=False, page=64, heads=4)
            ids = p.cache.table[0]
            p.cache.c[0, ids[where // 64].long(), where % 64, 5] = float("nan")
            V.mla_selftest_window_form(form)
            o = p.run()
            sees = torch.tensor([any(where in part for part in p.sees(0, i)) for i in range(new)])
            assert o[sees.cuda()][:, :, 5].isnan().all()
            rest = torch.ones(64, dtype=torch.bool)
            rest[5] = False
            assert not o[:, :, rest.cuda()].isnan()[sees.logical_not().cuda()].any()


@pytest.mark.parametrize("form", FORMS)
def test_score_ramps(form):
    """The running maximum grows from tile to tile and falls again."""
    for new in (1, 40):
        p = T.Problem([4000], [new], 2500, 300, dirty=False, turned=False, page=64, d_c=192 if new == 1 else 64)
        ramp = torch.linspace(-3, 3, 4000)[:, None].cuda()
        ids = p.cache.table[0][:63].long()
        rows = p.cache.c[0][ids].reshape(63 * 64, -1)
        rows[:4000, :1] = ramp * 8
        p.cache.c[0][ids] = rows.view(63, 64, -1)
        for size in (12.0, -12.0):
            p.q_c[:, :, 0] = size
            run(form, p, 6)


@pytest.mark.parametrize("form", FORMS)
@pytest.mark.parametrize("d_c", [64, 256])
def test_outputs_and_workspaces_off_32_bytes(form, d_c):
    p = T.Problem([500, 3000], [60, 1], 300, 20, heads=12, d_c=d_c, page=64, dirty=False)
    ref = run(form, p, 4)
    V.mla_selftest_window_form(form)
    p.workspace = torch.empty(p.workspace.numel() + 16, dtype=torch.uint8, device="cuda")[16:]
    o = torch.full((p.q_c.numel() + 8,), float("nan"), dtype=torch.bfloat16, device="cuda")
    assert o[8:].data_ptr() % 32 == 16
    p.call(o[8:].view(p.q_c.shape))
    torch.cuda.synchronize()
    assert torch.equal(o[8:].view(p.q_c.shape), ref) and o[:8].isnan().all()


@pytest.mark.parametrize("form", FORMS)
def test_bad_metadata_is_recorded(form):
    """Lengths, indices, page numbers and row starts that cannot be: nothing is read out of
    range, the other streams' rows are right, the refused ones' are left as they were."""
    for new in (1, 40):
        def fresh():
            return T.Problem([300, 200], [new, new], 100, 40, gone=[32, 0], heads=12, dirty=False)
        V.mla_selftest_window_form(form)
        ok = fresh()
        ref = ok.run()
        top = ok.cache.c[ok.cache.c.isfinite()].abs().max()
        for what in ("long", "negative", "gone", "far", "front", "page", "start"):
            p = fresh()
            rows = slice(new, 2 * new)
            if what == "long":
                p.cache.lens[0] = 1 << 20
            elif what == "negative":
                p.cache.lens[0] = -5
            elif what == "gone":
                p.win.dropped[0] = -16
            elif what == "far":
                p.win.dropped[0] = 2 ** 31 - 2 ** 16 - 100
            elif what == "front":
                p.cache.lens[0] = 40 + new - 1
            elif what == "page":
                p.cache.table[0, 17] = 1 << 20
            else:
                p.q_start[2] = 2 * new + 7
                rows = slice(0, new)
            o = p.run()
            assert V.mla_device_status(clear=True) == V.MLA_ERR_RANGE, what
            assert (o[rows].float() - ref[rows].float()).abs().max() <= 2 * T.REL * top, what
            if what not in ("page", "start"):
                assert o[:new].isnan().all(), what


def test_forms_in_a_graph():
    """A form is named when a call is captured; replays keep it, with lengths of their own."""
    for form in FORMS:
        p = T.Problem([900, 140], [1, 50], 300, 20, gone=[16, 0], heads=12, d_c=192, dirty=False)
        o, graph = torch.full_like(p.q_c, float("nan")), torch.cuda.CUDAGraph()
        V.mla_selftest_window_form(form)
        with torch.cuda.graph(graph):
            p.call(o)
        V.mla_selftest_window_form(0)
        for cut in (0, 7):
            p.lens = [k - cut for k in p.lens]
            p.cache.lens.sub_(cut)
            graph.replay()
            torch.cuda.synchronize()
            p.check(o, 5)


def test_the_choice():
    """What the estimates take: a team for one token, shares for a long window, tiles of 128 rows
    for prompts, pairs for chunks."""
    for lens, new, window, want in (([300], [1], 100, TEAMS), ([30000], [1], 20000, (SHARES,)),
                                    ([3000] * 9, [20] * 9, 2900, (TILES,)), ([3000] * 2, [2000] * 2, 900, (PAIRS,))):
        p = T.Problem(lens, new, window, 4, heads=12, d_c=64, page=64, dirty=False)
        p.run()
        assert V.mla_selftest_window_form(0) in want, lens


def test_forms_that_are_not_there():
    for bad in (-1, 3, 5, 32, 64, 512):
        with pytest.raises(V.MlaError):
            V.mla_selftest_window_form(bad)
    p = T.Problem([300], [1], 100, 4, d_c=512, dirty=False)
    o = torch.full_like(p.q_c, float("nan"))
    for form in (*TEAMS, SHARES, PAIRS):
        V.mla_selftest_window_form(form)
        with pytest.raises(V.MlaError):
            p.call(o)
    torch.cuda.synchronize()
    assert o.isnan().all() and V.mla_device_status(clear=True) == V.MLA_OK
