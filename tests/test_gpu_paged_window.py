"""Attention over the sinks and the sliding window of paged streams against the float64
oracle.

Tolerance per value: the weights are rounded to bf16 once (2^-8 of each) and the output
once (2^-8 of at most sum_j p_j |c_j|); fp32 scores of 96 .. 576 products, with the size
of the scores here, move a weight by less than 2^-10. So
|o - ref| <= (2 * 2^-8 + 2^-10) * sum_j p_j |c_j|."""

import math
import os
import subprocess
import sys

import numpy as np
import pytest
import torch

from oracle import paged_oracle as O
from paper_2605_30351_gb300 import videomla as V

pytestmark = pytest.mark.gpu

REL = 2 * 2.0 ** -8 + 2.0 ** -10
I32 = torch.int32


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    V.load()
    V.mla_device_status(clear=True)
    yield
    assert V.mla_device_status(clear=True) == V.MLA_OK


class Problem:
    """Streams that hold lens tokens, gave gone back and have new ones, in a pool whose
    other rows hold NaN and infinities; so do the held keys that no new token sees."""

    def __init__(self, lens, new, window, sinks, block=1, gone=None, turned=True, heads=4, d_c=64,
                 d_r=32, page=16, seed=0, gain=1.0, layers=1, dirty=True, spare=3):
        g = torch.Generator().manual_seed(seed)
        self.lens, self.new, self.block = list(lens), list(new), block
        self.gone = [0] * len(lens) if gone is None else list(gone)
        self.window, self.sinks, self.page, self.layer = window, sinks, page, layers - 1
        need = [-(-k // page) for k in lens]
        pages = sum(need) + spare
        place = torch.randperm(pages, generator=g)[:sum(need)].to(I32)
        table = torch.full((len(lens), max(need + [1]) + 1), -1, dtype=I32)
        c = torch.full((layers, pages, page, d_c), float("nan"))
        kr = torch.full((layers, pages, page, d_r), float("inf"))
        kr[:, :, ::2] = float("nan")
        at = 0
        for s, k in enumerate(lens):
            ids = place[at:at + need[s]]
            at += need[s]
            table[s, :need[s]] = ids
            seen = np.zeros(k, bool)
            for i in range(new[s]):
                for part in self.sees(s, i):
                    seen[part] = True
            a = torch.arange(k)
            if dirty:
                a = a[torch.from_numpy(seen)]
            c[layers - 1, ids[a // page].long(), a % page] = torch.randn(len(a), d_c, generator=g)
            kr[layers - 1, ids[a // page].long(), a % page] = torch.randn(len(a), d_r, generator=g)
        refs = torch.zeros(pages, dtype=I32)
        refs[place.long()] = 1
        self.cache = V.PagedCache(c.to(torch.bfloat16).cuda(), kr.to(torch.bfloat16).cuda(),
                                  table.cuda(), torch.tensor(lens, dtype=I32).cuda(), refs.cuda())
        self.win = V.PagedWindow(window, sinks, None if gone is None else
                                 torch.tensor(self.gone, dtype=I32).cuda())
        t = sum(new)
        std = gain * math.sqrt((128 - d_r) / d_c)
        bf = torch.bfloat16
        self.q_c = (torch.randn(t, heads, d_c, generator=g) * std).to(bf).cuda()
        self.q_r = (torch.randn(t, heads, d_r, generator=g) * gain).to(bf).cuda()
        self.q_sink = (torch.randn(t, heads, d_r, generator=g) * gain).to(bf).cuda() if turned else None
        self.q_start = torch.tensor(np.concatenate([[0], np.cumsum(new)]), dtype=I32).cuda()
        self.workspace = torch.empty(V.mla_paged_workspace_bytes(self.cache), dtype=torch.uint8,
                                     device="cuda")

    def sees(self, s, i):
        return O.window_sees(self.lens[s] - self.new[s] + i, self.lens[s], self.gone[s],
                             self.block, self.window, self.sinks, self.page)

    def call(self, o, stream=None):
        V.mla_paged_window_attention(self.cache, self.win, self.layer, self.q_c, self.q_r,
                                     self.q_sink, self.q_start, 128, self.block, self.workspace,
                                     o, stream=stream)

    def run(self, stream=None):
        o = torch.full_like(self.q_c, float("nan"))
        if stream is not None:
            stream.wait_stream(torch.cuda.current_stream())
        self.call(o, stream)
        torch.cuda.synchronize()
        return o

    def keys(self, s):
        a = np.arange(self.lens[s])
        ids = self.cache.table[s].cpu().numpy()[a // self.page]
        return (self.cache.c[self.layer].double().cpu().numpy()[ids, a % self.page],
                self.cache.kr[self.layer].double().cpu().numpy()[ids, a % self.page])

    def check(self, o, tokens=None):
        """All new tokens, or the first, last and some of each stream."""
        host = [None if q is None else q.double().cpu().numpy()
                for q in (self.q_c, self.q_r, self.q_sink, o)]
        q_c, q_r, q_sink, got = host[0], host[1], host[2] if self.q_sink is not None else host[1], host[3]
        at = 0
        for s, n in enumerate(self.new):
            if not n:
                continue
            c, kr = self.keys(s)
            pick = range(n) if tokens is None or n <= tokens else sorted(
                {0, n - 1} | set(np.random.default_rng(s).integers(0, n, tokens).tolist()))
            for i in pick:
                ref, size = O.attend_window(q_c[at + i], q_r[at + i], q_sink[at + i], c, kr,
                                            self.sees(s, i), 128)
                err = np.abs(got[at + i] - ref)
                assert (err <= REL * size).all(), (s, i, np.max(err / np.maximum(size, 1e-30)))
            at += n


def run_check(p, tokens=None):
    o = p.run()
    p.check(o, tokens)
    return o


@pytest.mark.parametrize("d_c", [64, 128, 192, 256, 512])
@pytest.mark.parametrize("d_r", [32, 64])
@pytest.mark.parametrize("page", [16, 64, 100])
@pytest.mark.parametrize("turned", [True, False])
def test_shapes(d_c, d_r, page, turned):
    """Every kernel instance: one token, an idle stream, pages that end inside a key tile,
    more rows than a row tile, streams shorter and longer than window and sinks."""
    run_check(Problem([1, 300, 77, 530, 129], [1, 30, 0, 5, 129], 90, 21, heads=12, d_c=d_c, d_r=d_r,
                      page=page, turned=turned, seed=d_c + page))


@pytest.mark.parametrize("d_c,d_r", [(64, 64), (128, 32), (192, 32), (256, 64), (512, 64)])
@pytest.mark.parametrize("turned", [True, False])
def test_single_tokens(d_c, d_r, turned):
    """Decoding: a token or two of many streams."""
    run_check(Problem([1, 40, 513, 300, 700, 64, 129, 1000], [1, 1, 1, 0, 1, 1, 1, 1], 200, 17,
                      gone=[0, 0, 32, 0, 64, 0, 0, 1600], heads=8, d_c=d_c, d_r=d_r, turned=turned))


@pytest.mark.parametrize("window", [1, 2, 15, 16, 17, 63, 64, 65, 127, 128, 129, 200, 1000, 1 << 30])
@pytest.mark.parametrize("sinks", [0, 1, 4, 64, 100, 130, 300, 1 << 30])
def test_window_edges(window, sinks):
    """Few rows (the 16-row kernel) and many (tensor memory), windows and sinks that end
    inside tiles, meet, overlap, or are longer than the stream."""
    run_check(Problem([400, 9, 131], [1, 1, 2], window, sinks, seed=window % 97 + sinks % 89))
    run_check(Problem([400, 9, 131], [90, 9, 33], window, sinks, seed=window % 89 + sinks % 97))


@pytest.mark.parametrize("block", [0, 1, 2, 7, 64, 100, 1 << 30])
@pytest.mark.parametrize("gone", [None, [48, 0, 160, 0]])
def test_blocks(block, gone):
    """No mask, token by token, blocks that end inside tiles and before the newest token's
    block does; blocks count from a stream's start, given back or not."""
    run_check(Problem([333, 200, 150, 1], [150, 200, 64, 1], 77, 30, block, gone=gone), 24)
    run_check(Problem([333, 200, 150, 1], [3, 1, 2, 1], 77, 30, block, gone=gone))


@pytest.mark.parametrize("page", [8, 24, 32, 48, 96, 120, 128, 200, 256])
@pytest.mark.parametrize("new", [2, 40])
def test_page_sizes(page, new):
    run_check(Problem([700, 3, 1700], [new, 2, new], 300, 130, gone=[page * 2, 0, page * 7], page=page,
                      heads=5), 9)


@pytest.mark.parametrize("heads", [1, 3, 16, 40, 128, 200])
@pytest.mark.parametrize("new", [1, 2, 17])
def test_head_counts(heads, new):
    run_check(Problem([260, 40], [new, new], 100, 12, heads=heads))


def test_rows_that_see_nothing():
    """More new tokens than the stream holds: the first of them have negative places and
    see no key; an empty stream's rows are 0 too."""
    run_check(Problem([3, 0, 130, 0], [9, 4, 140, 0], 20, 2, heads=12))
    run_check(Problem([0, 0], [1, 2], 20, 2, block=0))
    run_check(Problem([0], [1], 20, 0))
    run_check(Problem([4], [300], 2, 0, block=3))


@pytest.mark.parametrize("lens,new,window,sinks", [
    ([5000], [1], 3000, 64), ([30000], [2], 20000, 1000), ([3000] * 7, [1] * 7, 1500, 4),
    ([9001, 70, 1, 12011], [1, 1, 1, 3], 8000, 1560), ([9001, 70, 1, 12011], [1, 70, 1, 300], 4096, 200),
    ([6000], [6000], 700, 16)])
def test_long_streams(lens, new, window, sinks):
    """Few rows and many keys: work split along the keys and joined; a prompt much longer
    than its window."""
    p = Problem(lens, new, window, sinks, heads=12, d_c=192, page=64, seed=9,
                dirty=sum(new) < 1000)
    o = run_check(p, 4)
    assert torch.equal(o, p.run())                   # and the same again, bit for bit


@pytest.mark.parametrize("d_c,d_r", [(512, 64), (512, 32), (256, 64), (64, 32)])
def test_long_streams_other_widths(d_c, d_r):
    run_check(Problem([7003, 100, 2500], [2, 90, 40], 3000, 333, d_c=d_c, d_r=d_r, heads=16, page=32), 4)


@pytest.mark.parametrize("d_c,d_r", [(64, 32), (128, 64), (192, 32), (256, 64), (512, 32)])
@pytest.mark.parametrize("page", [16, 100])
def test_single_tokens_of_many_long_streams(d_c, d_r, page):
    """As many key blocks as share the work among all SMs, cut tiles joined by a second
    kernel; one stream has more rows than a tile."""
    n = 24
    p = Problem([4300 - 31 * s for s in range(n)], [3 if s == 5 else 1 for s in range(n)], 4000, 130,
                gone=[page * (s % 3) for s in range(n)], heads=12, d_c=d_c, d_r=d_r, page=page, seed=d_c)
    o = run_check(p)
    assert torch.equal(o, p.run())


@pytest.mark.parametrize("seqs,new,window", [(1, 40, 60), (3, 7, 300), (40, 2, 100), (150, 1, 100),
                                             (200, 1, 20), (9, 5, 1000)])
def test_teams(seqs, new, window):
    """Teams of one to eight CTAs, each with whole tiles: a stream's further tiles, more tiles
    than teams, streams that are idle."""
    rng = np.random.default_rng(seqs)
    counts = [new if s % 4 else int(rng.integers(0, 2 * new + 1)) for s in range(seqs)]
    counts[-1] = max(1, counts[-1])
    lens = [int(rng.integers(n, n + 1500)) for n in counts]
    for turned in (True, False):
        p = Problem(lens, counts, window, 20, heads=12, d_c=128, page=32, turned=turned, seed=window)
        o = run_check(p, 6)
        assert torch.equal(o, p.run())


def test_random_calls():
    """Sizes and masks drawn at random."""
    rng = np.random.default_rng(5)
    for k in range(40):
        seqs = int(rng.integers(1, 6))
        page = int(rng.choice([8, 16, 24, 64, 128]))
        sinks = int(rng.choice([0, 1, 5, 60, 200]))
        wide = rng.random() < 0.5
        front = O.front(sinks, page)
        new = [int(rng.integers(0, 60 if wide else 3)) for _ in range(seqs)]
        if sum(new) == 0:
            new[0] = 1
        gone = [int(rng.integers(0, 9)) * page for _ in range(seqs)]
        lens = [int(rng.integers(n + (front if g else 0), n + front + 500)) for n, g in zip(new, gone)]
        run_check(Problem(lens, new, int(rng.integers(1, 400)), sinks,
                          block=int(rng.choice([0, 1, 1, 3, 50])), gone=gone,
                          turned=bool(rng.random() < 0.6), heads=int(rng.choice([1, 4, 12])),
                          d_c=int(rng.choice([64, 128, 192, 256, 512])),
                          d_r=int(rng.choice([32, 64])), page=page, seed=k), 12)


def test_a_window_of_everything_is_plain_attention():
    for new in (1, 50):
        p = Problem([300, 77], [new, new], 1 << 30, 0, turned=False, heads=12, d_c=192)
        o, ref = p.run(), torch.empty_like(p.q_c)
        p.check(o)
        V.mla_paged_attention(p.cache, 0, p.q_c, p.q_r, p.q_start, 128, 1, p.workspace, ref)
        assert (o.float() - ref.float()).abs().max() <= 2 * REL * p.cache.c[p.cache.c.isfinite()].abs().max()


@pytest.mark.parametrize("block", [1, 0, 7])
def test_indices_near_their_limit(block):
    """Streams that went on for 2^31 tokens: blocks count from their start."""
    gone = ((2 ** 31 - 2 ** 16 - 500) // 16) * 16
    run_check(Problem([400, 300], [20, 1], 100, 20, block, gone=[gone, 16]))
    run_check(Problem([400, 300], [1, 1], 100, 20, block, gone=[gone, 16]))


@pytest.mark.parametrize("new", [1, 40])
def test_what_a_row_sees_reaches_it(new):
    """A NaN in a sink or window key that rows see reaches them, wherever the work is cut;
    an infinite score wins."""
    for where in (2, 5990):
        p = Problem([6000], [new], 3000, 16, dirty=False, page=64, heads=4)
        ids = p.cache.table[0]
        p.cache.c[0, ids[where // 64].long(), where % 64, 5] = float("nan")
        o = p.run()
        sees = torch.tensor([any(where in part for part in p.sees(0, i)) for i in range(new)])
        assert o[sees.cuda()][:, :, 5].isnan().all()
        rest = torch.ones(64, dtype=torch.bool)
        rest[5] = False
        assert not o[:, :, rest.cuda()].isnan()[sees.logical_not().cuda()].any()


def test_score_ramps():
    """The running maximum grows from tile to tile and falls again."""
    for new in (1, 40):
        p = Problem([4000], [new], 2500, 300, dirty=False, turned=False, page=64)
        ramp = torch.linspace(-3, 3, 4000)[:, None].cuda()
        ids = p.cache.table[0][:63].long()
        rows = p.cache.c[0][ids].reshape(-1, 64)
        rows[:4000, :1] = ramp * 8
        p.cache.c[0][ids] = rows.view(63, 64, 64)
        p.q_c[:, :, 0] = 12.0
        run_check(p, 6)
        p.q_c[:, :, 0] = -12.0
        run_check(p, 6)


def test_layers_and_offsets_past_4_gib():
    c = torch.zeros(3, 80000, 64, 192, dtype=torch.bfloat16, device="cuda")
    kr = torch.zeros(3, 80000, 64, 32, dtype=torch.bfloat16, device="cuda")
    g = torch.Generator(device="cuda").manual_seed(1)
    ids = torch.tensor([79990, 3, 79999, 40000, 79000, 77], dtype=I32, device="cuda")
    c[2, ids.long()] = torch.randn(6, 64, 192, device="cuda", generator=g).to(torch.bfloat16)
    kr[2, ids.long()] = torch.randn(6, 64, 32, device="cuda", generator=g).to(torch.bfloat16)
    small = Problem([380, 380], [30, 30], 150, 70, heads=12, d_c=192, page=64, dirty=False)
    for new in (30, 1):
        p = Problem([380], [new], 150, 70, heads=12, d_c=192, page=64, dirty=False)
        refs = torch.ones(80000, dtype=I32, device="cuda")
        p.cache = V.PagedCache(c, kr, torch.nn.functional.pad(ids[None], (0, 1), value=-1), p.cache.lens, refs)
        p.layer = 2
        k = c[2, ids.long()].reshape(-1, 192)[:380].double().cpu().numpy()
        r = kr[2, ids.long()].reshape(-1, 32)[:380].double().cpu().numpy()
        p.keys = lambda s: (k, r)
        run_check(p, 5)
    del small


def test_many_streams():
    """More streams than the share search has threads, most of them idle."""
    seqs = 700
    lens = [(37 * s) % 300 + 10 for s in range(seqs)]
    new = [3 if s % 5 == 0 else 0 for s in range(seqs)]
    run_check(Problem(lens, new, 100, 10, gone=[16 * (s % 4) if lens[s] > 30 else 0 for s in range(seqs)],
                      heads=12))
    new = [150 if s in (3, 650) else 0 for s in range(seqs)]
    lens[3], lens[650] = 500, 460
    run_check(Problem(lens, new, 100, 10, heads=12), 9)


def test_other_stream_and_graph():
    """Another stream; two captured graphs with a workspace each, replayed in turn with
    other lengths and queries in place."""
    ps = [Problem([300, 40], [1, 1], 100, 20, gone=[16, 0], heads=12, d_c=192, dirty=False),
          Problem([300, 140], [40, 50], 100, 20, gone=[16, 0], heads=12, d_c=192, dirty=False)]
    side = torch.cuda.Stream()
    graphs = []
    for p in ps:
        p.check(p.run(side))
        o, graph = torch.full_like(p.q_c, float("nan")), torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            p.call(o)
        graphs.append((p, graph, o))
    for cut in (0, 7):
        for p, graph, o in graphs:
            p.lens = [k - cut for k in p.lens]
            p.cache.lens.sub_(cut)
            p.q_c.mul_(0.5)
        for _, graph, _ in graphs:
            graph.replay()
        torch.cuda.synchronize()
        for p, _, o in graphs:
            p.check(o)


def test_dirty_workspace():
    for new in (1, 30):
        p = Problem([5000, 200], [new, new], 3000, 100, heads=12, page=64, dirty=False)
        ref = p.run()
        p.workspace.fill_(255)
        assert torch.equal(ref, p.run())


def test_an_unaligned_workspace():
    p = Problem([5000, 200], [1, 30], 3000, 100, heads=12, page=64, dirty=False)
    ref = p.run()
    p.workspace = torch.empty(p.workspace.numel() + 16, dtype=torch.uint8, device="cuda")[16:]
    assert torch.equal(ref, p.run())


@pytest.mark.parametrize("new", [[2], [60], [400]])
@pytest.mark.parametrize("d_c", [64, 192, 256, 512])
def test_an_output_off_32_bytes(new, d_c):
    """o on a 16-byte boundary: rows are not stored 32 bytes at a time."""
    p = Problem([500], new, 100, 20, heads=12, d_c=d_c, page=64, dirty=False)
    ref = p.run()
    o = torch.full((p.q_c.numel() + 8,), float("nan"), dtype=torch.bfloat16, device="cuda")
    assert o[8:].data_ptr() % 32 == 16
    p.call(o[8:].view(p.q_c.shape))
    torch.cuda.synchronize()
    assert torch.equal(o[8:].view(p.q_c.shape), ref) and o[:8].isnan().all()


def test_bad_metadata_is_recorded():
    """Lengths, indices, page numbers and row starts that cannot be: nothing is read out of
    range, the other streams' rows are right."""
    for new in (1, 40):
        def fresh():
            return Problem([300, 200], [new, new], 100, 40, gone=[32, 0], heads=12, dirty=False)
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
            elif what == "front":                     # new tokens among the sinks' pages
                p.cache.lens[0] = 40 + new - 1
            elif what == "page":
                p.cache.table[0, 17] = 1 << 20
            else:
                p.q_start[2] = 2 * new + 7
                rows = slice(0, new)
            o = p.run()
            assert V.mla_device_status(clear=True) == V.MLA_ERR_RANGE, what
            ok = fresh()
            ref = ok.run()
            err = (o[rows].float() - ref[rows].float()).abs().max()
            assert err <= 2 * REL * ok.cache.c[ok.cache.c.isfinite()].abs().max(), what
            if what not in ("page", "start"):
                assert o[:new].isnan().all(), what    # not written
    assert V.mla_device_status(clear=True) == V.MLA_OK


def test_refusals():
    p = Problem([30], [2], 10, 4, dirty=False)
    o = torch.empty_like(p.q_c)

    def call(**kw):
        a = dict(cache=p.cache, window=p.win, layer=0, q_c=p.q_c, q_r=p.q_r, q_r_sink=p.q_sink,
                 q_start=p.q_start, head_dim=128, causal_block=1, workspace=p.workspace, o=o)
        a.update(kw)
        V.mla_paged_window_attention(**a)

    call()
    with pytest.raises(TypeError):
        call(q_r_sink=p.q_sink.float())
    with pytest.raises(ValueError):
        call(q_r_sink=p.q_sink[:1])
    with pytest.raises(ValueError):
        call(window=V.PagedWindow(10, 4, torch.zeros(2, dtype=I32, device="cuda")))
    with pytest.raises(TypeError):
        V.PagedWindow(10, 4, torch.zeros(2, device="cuda"))
    for bad in (V.PagedWindow(0, 4), V.PagedWindow(-1), V.PagedWindow(3, -1)):
        with pytest.raises(V.MlaError):
            call(window=bad)
    with pytest.raises(V.MlaError):
        call(workspace=p.workspace[:-16])
    pinned = torch.zeros(1, dtype=I32).pin_memory()
    w = V.PagedWindow(10, 4)
    w.struct.dropped = pinned.data_ptr()
    with pytest.raises(V.MlaError):
        call(window=w)
    torch.cuda.synchronize()
    assert V.mla_device_status(clear=True) == V.MLA_OK


def test_two_streams_at_once():
    """Calls that overlap on the GPU, a workspace each."""
    ps = [Problem([3000, 40, 700], [1, 1, 1], 2000, 20, heads=12, d_c=192, page=64, dirty=False, seed=1),
          Problem([900, 140], [60, 70], 300, 20, heads=12, d_c=192, page=64, dirty=False, seed=2),
          Problem([4100 - 9 * s for s in range(20)], [1] * 20, 4000, 20, heads=12, page=64, dirty=False, seed=3)]
    streams = [torch.cuda.Stream() for _ in ps]
    outs = [torch.full_like(p.q_c, float("nan")) for p in ps]
    torch.cuda.synchronize()
    for _ in range(20):
        for p, o, s in zip(ps, outs, streams):
            p.call(o, s)
    torch.cuda.synchronize()
    for p, o in zip(ps, outs):
        p.check(o, 5)
        assert torch.equal(o, p.run())


FIRST = """
import sys
sys.path[:0] = [{root!r}, {here!r}]
import torch
import test_gpu_paged_window as T
for lens, new, window in (([300], [1], 100), ([4100] * 20, [1] * 20, 4000), ([300, 90], [40, 30], 100)):
    p = T.Problem(lens, new, window, 20, heads=12, d_c=192, page=64, dirty=False)
    o, graph = torch.full_like(p.q_c, float("nan")), torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        p.call(o)
    graph.replay()
    torch.cuda.synchronize()
    p.check(o, 4)
assert T.V.mla_device_status(clear=True) == T.V.MLA_OK
print("first calls ok")
"""


def test_first_calls_inside_a_capture():
    """A process whose first call of every form is captured."""
    here = os.path.dirname(os.path.abspath(__file__))
    code = FIRST.format(root=os.path.dirname(here), here=here)
    r = subprocess.run([sys.executable, "-c", code], capture_output=True, text=True, timeout=300)
    assert r.returncode == 0 and "first calls ok" in r.stdout, r.stdout + r.stderr
