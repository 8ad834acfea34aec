"""Sliding, step plans and positions of paged streams against the oracle's rules, integer
for integer, and whole steps of them together against the framework's sink ring."""

import numpy as np
import pytest
import torch

from oracle import paged_oracle as O
from paper_2605_30351_gb300 import synth
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


def host(t):
    return t.cpu().numpy()


def pool(tokens=8, seqs=6, pages=61, max_pages=12, sinks=0, window=20):
    cache = V.PagedCache.empty(2, pages, tokens, seqs, max_pages, 64, 32)
    win = V.PagedWindow(window, sinks, torch.zeros(seqs, dtype=I32, device="cuda"))
    return cache, win, O.Pages(2, pages, tokens, seqs, max_pages, 64, 32), np.zeros(seqs, np.int64)


def same(cache, win, o, gone):
    assert np.array_equal(host(cache.table), o.table)
    assert np.array_equal(host(cache.lens), o.lens)
    assert np.array_equal(host(cache.refs), o.refs)
    assert np.array_equal(host(win.dropped), gone)


@pytest.mark.parametrize("seed,tokens,seqs,sinks", [(1, 8, 6, 0), (2, 16, 3, 5), (3, 24, 11, 24),
                                                    (4, 8, 40, 17)])
def test_random_operations(seed, tokens, seqs, sinks):
    """Plan, grow, slide, branch, end and pack in random order."""
    cache, win, o, gone = pool(tokens, seqs, 200, 12, sinks)
    rng = np.random.default_rng(seed)
    for _ in range(60):
        kind = rng.integers(5)
        if kind <= 1:
            n = np.where(rng.random(seqs) < 0.5, rng.integers(0, 3 * tokens, seqs), 0)
            n = np.where(o.lens + n > 12 * tokens, 0, n)
            q_start = torch.empty(seqs + 1, dtype=I32, device="cuda")
            new_lens = torch.empty(seqs, dtype=I32, device="cuda")
            V.mla_paged_window_plan(cache, win, i32(n), q_start, new_lens)
            gone[o.lens == 0] = 0
            assert np.array_equal(host(q_start), np.concatenate([[0], np.cumsum(n)]))
            want = np.where(n > 0, o.lens + n, -1)
            assert np.array_equal(host(new_lens), want)
            V.mla_pages_resize(cache, new_lens)
            o.resize(want)
        elif kind == 2:
            keep = np.where(rng.random(seqs) < 0.3, -1, rng.integers(0, 5 * tokens, seqs))
            V.mla_pages_slide(cache, win, i32(keep))
            O.slide(o, gone, keep, sinks)
        elif kind == 3:
            ends = np.where(rng.random(seqs) < 0.2, 0, -1)
            V.mla_pages_resize(cache, i32(ends))
            o.resize(ends)
        else:
            held, empty = np.flatnonzero(o.lens > 0), np.flatnonzero(o.lens == 0)
            n = min(len(held), len(empty))
            if n:
                src, dst = rng.permutation(held)[:n], rng.permutation(empty)[:n]
                V.mla_pages_window_fork(cache, win, i32(src), i32(dst))
                o.fork(src, dst)
                gone[dst] = gone[src]
        assert V.mla_device_status(clear=True) == (V.MLA_ERR_RANGE if o.range_error else V.MLA_OK)
        o.range_error = False
        same(cache, win, o, gone)


@pytest.mark.parametrize("sinks", [0, 1, 8, 9, 50])
@pytest.mark.parametrize("keep", [0, 1, 7, 8, 9, 40, 1 << 30])
def test_slide_edges(sinks, keep):
    """Lengths from nothing to a full list, whole pages and not."""
    lens = [0, 1, 7, 8, 9, 15, 16, 17, 40, 63, 64, 95, 96]
    cache, win, o, gone = pool(8, len(lens), 100, 12, sinks)
    V.mla_pages_resize(cache, i32(lens))
    o.resize(lens)
    for _ in range(2):                                # the second time nothing is left to go
        V.mla_pages_slide(cache, win, i32([keep] * len(lens)))
        O.slide(o, gone, [keep] * len(lens), sinks)
        same(cache, win, o, gone)


def test_slide_long_lists():
    """Lists of thousands of pages, moved by less and by more than a block's threads."""
    rng = np.random.default_rng(3)
    for n in (1, 100, 255, 256, 257, 3000):
        cache, win, o, gone = pool(8, 3, 12000, 4000, 20)
        lens = [8 * 4000, 8 * (n + 3) + 5, int(rng.integers(1, 8 * 4000))]
        V.mla_pages_resize(cache, i32(lens))
        o.resize(lens)
        keep = [8 * (4000 - 3 - n), 3, 9]
        V.mla_pages_slide(cache, win, i32(keep))
        O.slide(o, gone, keep, 20)
        same(cache, win, o, gone)


def test_branches_keep_their_pages():
    cache, win, o, gone = pool(8, 3, 40, 12, 8)
    for op in (lambda: (V.mla_pages_resize(cache, i32([60, 0, -1])), o.resize([60, 0, -1])),
               lambda: (V.mla_pages_window_fork(cache, win, i32([0]), i32([1])), o.fork([0], [1])),
               lambda: (V.mla_pages_slide(cache, win, i32([20, -1, -1])), O.slide(o, gone, [20, -1, -1], 8))):
        op()
        same(cache, win, o, gone)
    assert (host(cache.refs)[o.table[1][o.table[1] >= 0]] >= 1).all()


def test_slide_bad_metadata():
    """A length past the list, a negative count, indices past their limit: left alone and
    recorded; a page number outside the pool leaves the list and is recorded."""
    for what in ("long", "negative", "gone", "far", "page"):
        cache, win, o, gone = pool(8, 2, 40, 12)
        V.mla_pages_resize(cache, i32([60, 60]))
        o.resize([60, 60])
        if what == "long":
            cache.lens[0] = 97
        elif what == "negative":
            cache.lens[0] = -1
        elif what == "gone":
            win.dropped[0] = -8
        elif what == "far":
            win.dropped[0] = 2 ** 31 - 2 ** 16 - 60
        else:
            cache.table[0, 2] = 99
        before = [t.clone() for t in (cache.lens, win.dropped, cache.table)]
        V.mla_pages_slide(cache, win, i32([20, 20]))
        assert V.mla_device_status(clear=True) == V.MLA_ERR_RANGE, what
        for t, b in zip((cache.lens, win.dropped, cache.table), before):
            if what != "page":
                assert torch.equal(t[0], b[0]), what
        O.slide(o, gone, [-1, 20], 0)
        assert np.array_equal(host(cache.table)[1], o.table[1]) and int(cache.lens[1]) == o.lens[1]


@pytest.mark.parametrize("seqs", [1, 31, 32, 33, 1023, 1024, 1025, 5000, 65536])
def test_plan(seqs):
    rng = np.random.default_rng(seqs)
    cache = V.PagedCache.empty(1, 8, 8, seqs, 4, 8, 8)
    lens, n = rng.integers(0, 3, seqs) * 9, rng.integers(0, 4, seqs) * rng.integers(0, 2, seqs) * 7
    gone = rng.integers(0, 5, seqs) * 8
    cache.lens.copy_(i32(lens))
    win = V.PagedWindow(5, 1, i32(gone))
    q_start, new_lens = i32(np.full(seqs + 1, -7)), i32(np.full(seqs, -7))
    V.mla_paged_window_plan(cache, win, i32(n), q_start, new_lens)
    assert np.array_equal(host(q_start), np.concatenate([[0], np.cumsum(n)]))
    assert np.array_equal(host(new_lens), np.where(n > 0, lens + n, -1))
    assert np.array_equal(host(win.dropped), np.where(lens == 0, 0, gone))
    V.mla_paged_window_plan(cache, V.PagedWindow(5, 1), i32(n), q_start, new_lens)
    assert np.array_equal(host(q_start), np.concatenate([[0], np.cumsum(n)]))
    assert V.mla_device_status(clear=True) == V.MLA_OK


def test_plan_bad_counts():
    cache = V.PagedCache.empty(1, 8, 8, 4, 4, 8, 8)
    q_start, new_lens = i32([9] * 5), i32([9] * 4)
    V.mla_paged_window_plan(cache, V.PagedWindow(5), i32([3, -2, 0, 4]), q_start, new_lens)
    assert V.mla_device_status(clear=True) == V.MLA_ERR_RANGE
    assert host(q_start).tolist() == [0, 3, 3, 3, 7] and host(new_lens).tolist() == [3, -1, -1, 4]
    V.mla_paged_window_plan(cache, V.PagedWindow(5), i32([2 ** 31 - 1, 5, 0, 4]), q_start, new_lens)
    assert V.mla_device_status(clear=True) == V.MLA_ERR_RANGE
    assert host(q_start).tolist() == [0] + [2 ** 31 - 1] * 4


@pytest.mark.parametrize("axes,frame,width", [(3, 1560, 52), (3, 64, 8), (1, 1, 1), (1, 5, 2), (3, 7, 7)])
@pytest.mark.parametrize("block", [0, 1, 60])
@pytest.mark.parametrize("gone", [True, False])
def test_positions(axes, frame, width, block, gone):
    page, sinks, window = 16, 20, 90
    lens, new = [400, 33, 0, 17, 900, 64], [100, 33, 0, 1, 1, 0]
    back = [160, 0, 0, 0, 2 ** 31 - 2 ** 16 - 912, 0] if gone else [0] * 6
    g = torch.Generator().manual_seed(1)
    table = torch.full((6, 60), -1, dtype=I32)
    ids, at = torch.randperm(120, generator=g).to(I32), 0
    for s, k in enumerate(lens):
        m = -(-k // page)
        table[s, :m] = ids[at:at + m]
        at += m
    cache = V.PagedCache(torch.zeros(1, 120, page, 8, dtype=BF16, device="cuda"),
                         torch.zeros(1, 120, page, 8, dtype=BF16, device="cuda"), table.cuda(),
                         i32(lens), torch.ones(120, dtype=I32, device="cuda"))
    win = V.PagedWindow(window, sinks, i32(back) if gone else None)
    total = sum(new)
    pos, sink, rows = (torch.full(s, -9, dtype=I32, device="cuda") for s in
                       ((total, axes), (total, axes), (total,)))
    q_start = i32(np.concatenate([[0], np.cumsum(new)]))
    V.mla_paged_window_positions(cache, win, q_start, block, frame, width, pos, sink, rows)
    want, beside, at = [], [], []
    for s, (k, b, n) in enumerate(zip(lens, back, new)):
        x, y = O.window_positions(k, b, n, block, window, sinks, frame, width)
        want += x
        beside += y
        at += [int(table[s, p // page]) * page + p % page for p in range(k - n, k)]
    assert np.array_equal(host(pos), np.array(want)[:, :axes])
    assert np.array_equal(host(sink), np.array(beside)[:, :axes])
    assert np.array_equal(host(rows), at)
    again = torch.full_like(pos, -9)
    V.mla_paged_window_positions(cache, win, q_start, block, frame, width, again)
    assert torch.equal(again, pos)
    assert V.mla_device_status(clear=True) == V.MLA_OK


def test_positions_of_many_streams():
    """Streams of none, one and many tokens inside one block of threads, more streams than
    threads."""
    rng = np.random.default_rng(2)
    new = rng.integers(0, 3, 2000) * rng.integers(0, 2, 2000)
    new[5], new[1999] = 700, 300
    lens = np.where(new > 0, new + rng.integers(0, 9, 2000), 0)
    cache = V.PagedCache.empty(1, 4000, 8, 2000, 100, 8, 8)
    V.mla_pages_resize(cache, i32(lens))
    total = int(new.sum())
    pos, rows = torch.full((total, 1), -9, dtype=I32, device="cuda"), torch.full((total,), -9, dtype=I32, device="cuda")
    V.mla_paged_window_positions(cache, V.PagedWindow(9), i32(np.concatenate([[0], np.cumsum(new)])), 1, 1, 1,
                                 pos, None, rows)
    table = host(cache.table)
    p = np.concatenate([np.arange(k - n, k) for k, n in zip(lens, new)])
    s = np.repeat(np.arange(2000), new)
    assert np.array_equal(host(pos)[:, 0], p)
    assert np.array_equal(host(rows), table[s, p // 8] * 8 + p % 8)


def test_positions_bad_metadata():
    cache = V.PagedCache.empty(1, 8, 8, 2, 4, 8, 8)
    V.mla_pages_resize(cache, i32([20, 9]))
    win = V.PagedWindow(5, 0, i32([0, 0]))

    def call(q):
        pos, rows = torch.full((6, 3), -9, dtype=I32, device="cuda"), torch.full((6,), -9, dtype=I32, device="cuda")
        V.mla_paged_window_positions(cache, win, i32(q), 1, 4, 2, pos, None, rows)
        return host(pos), host(rows), V.mla_device_status(clear=True)

    pos, rows, st = call([0, 3, 6])
    assert st == V.MLA_OK and (pos >= 0).all() and (rows >= 0).all()
    for q, untouched in (([0, 3, 5], [5]), ([0, 3, 9], [3, 4, 5]), ([1, 3, 6], [0]), ([0, 4, 3], [])):
        pos, rows, st = call(q)
        assert st == V.MLA_ERR_RANGE, q
        assert (rows[untouched] == -9).all() and (pos[untouched] == -9).all(), q
    cache.table[1, 0] = 77
    pos, rows, st = call([0, 3, 6])
    assert st == V.MLA_ERR_RANGE and rows[3:].tolist()[0] == -1 and (rows[:3] >= 0).all()
    cache.lens[0] = 2                                  # the first new token at place -1
    pos, rows, st = call([0, 3, 6])
    assert st == V.MLA_ERR_RANGE and rows[0] == -1 and (pos[0] == 0).all() and rows[1] >= 0
    win.dropped[0] = 2 ** 31 - 1
    pos, rows, st = call([0, 3, 6])
    assert st == V.MLA_ERR_RANGE and (rows[:3] == -1).all() and (pos[:3] == 0).all()


class Rollouts:
    """One attention layer of paged rollouts with sinks and a window, step by step."""

    def __init__(self, w, seqs, page=16):
        self.w, self.T = w, w.tokens_per_frame
        self.cfg = V.make_config(w)
        pages = -(-w.slots // page) + -(-self.T // page) + 4
        self.cache = V.PagedCache.empty(1, pages * seqs, page, seqs, pages, w.d_c, w.d_r)
        S, W = w.sink_frames, w.window_frames
        self.win = V.PagedWindow((W - S) * self.T, S * self.T, torch.zeros(seqs, dtype=I32, device="cuda"))
        self.rope = V.Rope(torch.from_numpy(V.mla_rope_table_fill(self.cfg)).cuda(), w.rope_pairs)
        self.ws = torch.empty(V.mla_paged_workspace_bytes(self.cache), dtype=torch.uint8, device="cuda")

    def step(self, n_new, c, kr, q_c, q_r, block, slide=True):
        """All of a step's calls on the stream, nothing read back."""
        w, seqs, total = self.w, self.cache.seqs, c.shape[0]
        q_start, new_lens = torch.empty(seqs + 1, dtype=I32, device="cuda"), torch.empty(seqs, dtype=I32, device="cuda")
        pos, sink = torch.empty(total, 3, dtype=I32, device="cuda"), torch.empty(total, 3, dtype=I32, device="cuda")
        q_sink, o = torch.empty_like(q_r), torch.full_like(q_c, float("nan"))
        V.mla_paged_window_plan(self.cache, self.win, n_new, q_start, new_lens)
        V.mla_pages_resize(self.cache, new_lens)
        V.mla_paged_window_positions(self.cache, self.win, q_start, block, self.T, w.grid_w, pos, sink)
        V.mla_paged_append(self.cache, 0, c, kr, q_start, pos, self.rope)
        V.mla_rope_apply(self.rope, q_r, sink, q_sink)
        V.mla_rope_apply(self.rope, q_r, pos, q_r)
        V.mla_paged_window_attention(self.cache, self.win, 0, q_c, q_r, q_sink, q_start, w.head_dim, block, self.ws, o)
        if slide:
            keep = torch.full((seqs,), self.win.window - block, dtype=I32, device="cuda")
            V.mla_pages_slide(self.cache, self.win, keep)
        return o


def ring_step(w, ring, q_c, q_r, first, frames):
    pos = synth.grid_positions(w, first, frames).cuda()
    nq = q_c.shape[0]
    ws = torch.empty(V.mla_window_workspace_bytes(ring.cfg, nq), dtype=torch.uint8, device="cuda")
    o = torch.empty(1, nq, w.heads, w.d_c, dtype=BF16, device="cuda")
    V.mla_attention_window_forward(ring, q_c[None], q_r[None], pos, synth.frame_coords(w).cuda(), ws, o)
    return o[0]


@pytest.mark.parametrize("frames,sinks,window", [(1, 1, 5), (2, 1, 5), (2, 2, 6)])
def test_rollouts_equal_the_sink_ring(frames, sinks, window):
    """Two rollouts, one a chunk ahead, over many chunks: the paged cache stays short and
    gives what the ring with sink frames and window-relative rotation gives. Both are within
    1e-2 (relative norm) of the float64 layer, the bound of the ring's own tests, so within
    2e-2 of each other."""
    w = synth.workload("tiny", batch=1).with_(batch=1, sink_frames=sinks, window_frames=window)
    T, n = w.tokens_per_frame, frames * w.tokens_per_frame
    wt = {k: v.cuda() for k, v in synth.draw_layer_weights(w, 3).items()}
    both = Rollouts(w, 2)
    rings = [V.LatentCache(V.make_config(w)) for _ in range(2)]
    done, longest = [0, 0], 0
    for step in range(9):
        run = [0] if step == 0 else [0, 1]
        stage, q = [], []
        for s in run:
            x = synth.draw_tokens(w, n, 100 * s + done[s]).cuda()
            V.mla_cache_append(rings[s], x, wt["w_dkv"], wt["gamma_kv"], wt["w_kr"], None, done[s], frames)
            st = V.LatentCache(V.make_config(w.with_(window_frames=frames, sink_frames=0), V.MLA_FLAG_ROTATE_AT_USE))
            V.mla_cache_append(st, x, wt["w_dkv"], wt["gamma_kv"], wt["w_kr"], None, 0, frames)
            stage.append((st.c[0], st.kr[0]))
            q.append(synth.draw_queries(w, n, 50 * s + step))
        q_c, q_r = (torch.cat([v[k][0] for v in q]).cuda() for k in (0, 1))
        want = [ring_step(w, rings[s], q_c[i * n:(i + 1) * n], q_r[i * n:(i + 1) * n], done[s], frames)
                for i, s in enumerate(run)]
        o = both.step(i32([n if s in run else 0 for s in range(2)]), torch.cat([v[0] for v in stage]),
                      torch.cat([v[1] for v in stage]), q_c, q_r, n)
        ref = torch.cat(want).float()
        assert ((o.float() - ref).norm() / ref.norm()).item() <= 2e-2, step
        for s in run:
            done[s] += frames
        longest = max(longest, int(both.cache.lens.max()))
    assert host(both.cache.lens + both.win.dropped).tolist() == [d * T for d in done]
    assert longest <= (window + sinks) * T
    assert V.mla_device_status(clear=True) == V.MLA_OK


def test_a_captured_step_goes_on_for_ever():
    """One graph of a whole step, replayed: every length, page and position comes from the
    device, and results equal those of calls in turn, bit for bit. A third stream ends and
    starts anew between replays."""
    w = synth.workload("tiny", batch=1).with_(batch=1, sink_frames=1, window_frames=3)
    g = torch.Generator(device="cuda").manual_seed(4)

    def rows(*shape):
        return torch.randn(*shape, device="cuda", generator=g).to(BF16)

    total = 3
    a, b = Rollouts(w, 3), Rollouts(w, 3)
    ins = [torch.empty(total, w.d_c, dtype=BF16, device="cuda"), torch.empty(total, w.d_r, dtype=BF16, device="cuda"),
           torch.empty(total, w.heads, w.d_c, dtype=BF16, device="cuda"),
           torch.empty(total, w.heads, w.d_r, dtype=BF16, device="cuda")]
    n_new = i32([1, 1, 1])
    for t in ins:
        t.zero_()
    b.step(n_new, *ins, 1)                            # loads every kernel before the capture
    V.mla_pages_resize(b.cache, i32([0, 0, 0]))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        o = b.step(n_new, *ins, 1)
    V.mla_pages_resize(b.cache, i32([0, 0, 0]))
    for step in range(300):
        fresh = [rows(*t.shape) for t in ins]
        for t, f in zip(ins, fresh):
            t.copy_(f)
        if step == 200:
            for r in (a, b):
                V.mla_pages_resize(r.cache, i32([-1, -1, 0]))
        graph.replay()
        ref = a.step(n_new, *fresh, 1)
        if step % 37 == 0 or step > 290:
            assert torch.equal(o, ref), step
    for t, u in ((a.cache.lens, b.cache.lens), (a.cache.table, b.cache.table), (a.win.dropped, b.win.dropped),
                 (a.cache.refs, b.cache.refs)):
        assert torch.equal(t, u)
    assert host(a.cache.lens + a.win.dropped).tolist() == [300, 300, 100]
    assert V.mla_device_status(clear=True) == V.MLA_OK
