"""Attention over the paged latent cache against the float64 oracle.

Tolerance per value: the weights are rounded to bf16 once (2^-8 of each) and
the output once (2^-8 of at most sum_j p_j |c_j|); fp32 scores of 224 .. 576
products, with the size of the scores here, move a weight by less than 2^-10.
So |o - ref| <= (2 * 2^-8 + 2^-10) * sum_j p_j |c_j|."""

import math

import numpy as np
import pytest
import torch

from oracle import paged_oracle as O
from paper_2605_30351_gb300 import videomla as V

pytestmark = pytest.mark.gpu

REL = 2 * 2.0 ** -8 + 2.0 ** -10


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    V.load()
    V.mla_device_status(clear=True)
    yield
    assert V.mla_device_status(clear=True) == V.MLA_OK


class Problem:
    """Streams of the given lengths and new tokens in a pool whose other rows
    hold NaN and infinities."""

    def __init__(self, lens, new, heads=12, d_c=192, d_r=32, page=64, seed=0, gain=1.0,
                 head_dim=128, layers=1, spare=3):
        g = torch.Generator().manual_seed(seed)
        self.lens, self.new, self.head_dim = list(lens), list(new), head_dim
        need = [-(-k // page) for k in lens]
        pages = sum(need) + spare
        place = torch.randperm(pages, generator=g)[:sum(need)].to(torch.int32)
        self.max_pages = max(need + [1]) + 1
        table = torch.full((len(lens), self.max_pages), -1, dtype=torch.int32)
        c = torch.full((layers, pages, page, d_c), float("nan"))
        kr = torch.full((layers, pages, page, d_r), float("inf"))
        kr[:, :, ::2] = float("nan")
        at = 0
        for s, k in enumerate(lens):
            ids = place[at:at + need[s]]
            at += need[s]
            table[s, :need[s]] = ids
            a = torch.arange(k)
            c[layers - 1, ids[a // page].long(), a % page] = torch.randn(k, d_c, generator=g)
            kr[layers - 1, ids[a // page].long(), a % page] = torch.randn(k, d_r, generator=g)
        refs = torch.zeros(pages, dtype=torch.int32)
        refs[place.long()] = 1
        self.layer = layers - 1
        self.cache = V.PagedCache(c.to(torch.bfloat16).cuda(), kr.to(torch.bfloat16).cuda(),
                                  table.cuda(), torch.tensor(lens, dtype=torch.int32).cuda(),
                                  refs.cuda())
        t = sum(new)
        std = gain * math.sqrt((head_dim - d_r) / d_c)
        self.q_c = (torch.randn(t, heads, d_c, generator=g) * std).to(torch.bfloat16).cuda()
        self.q_r = (torch.randn(t, heads, d_r, generator=g) * gain).to(torch.bfloat16).cuda()
        self.q_start = torch.tensor(np.concatenate([[0], np.cumsum(new)]),
                                    dtype=torch.int32).cuda()
        self.workspace = torch.empty(V.mla_paged_workspace_bytes(self.cache), dtype=torch.uint8,
                                     device="cuda")

    def run(self, block=1, stream=None):
        o = torch.full_like(self.q_c, float("nan"))
        if stream is not None:
            stream.wait_stream(torch.cuda.current_stream())
        V.mla_paged_attention(self.cache, self.layer, self.q_c, self.q_r, self.q_start,
                              self.head_dim, block, self.workspace, o, stream=stream)
        torch.cuda.synchronize()
        return o

    def keys(self, s):
        p = self.cache.c.shape[2]
        a = np.arange(self.lens[s])
        ids = self.cache.table[s].cpu().numpy()[a // p]
        return (self.cache.c[self.layer].double().cpu().numpy()[ids, a % p],
                self.cache.kr[self.layer].double().cpu().numpy()[ids, a % p])

    def check(self, o, block=1, tokens=None):
        """All new tokens, or the first, last and some of each stream."""
        at = 0
        for s, n in enumerate(self.new):
            if not n:
                continue
            c, kr = self.keys(s)
            pick = range(n) if tokens is None or n <= tokens else sorted(
                {0, n - 1} | set(np.random.default_rng(s).integers(0, n, tokens).tolist()))
            for i in pick:
                held, place = self.lens[s], self.lens[s] - n + i
                k = O.visible(place, held, block)
                got = o[at + i].double().cpu().numpy()
                if k == 0:
                    assert (got == 0).all(), (s, i)
                    continue
                q_c = self.q_c[at + i].double().cpu().numpy()
                q_r = self.q_r[at + i].double().cpu().numpy()
                x = (q_c @ c[:k].T + q_r @ kr[:k].T) / math.sqrt(self.head_dim)
                w = np.exp(x - x.max(-1, keepdims=True))
                w /= w.sum(-1, keepdims=True)
                err = np.abs(got - w @ c[:k])
                bound = REL * (w @ np.abs(c[:k]))
                assert (err <= bound).all(), (s, i, np.max(err / bound))
            at += n


def run_check(p, block=1, tokens=None):
    o = p.run(block)
    p.check(o, block, tokens)
    return o


@pytest.mark.parametrize("d_c", [64, 128, 192, 256, 512])
@pytest.mark.parametrize("d_r", [32, 64])
@pytest.mark.parametrize("page", [16, 64, 100])
def test_shapes(d_c, d_r, page):
    """Every kernel instance, ragged streams: one token, an idle stream, pages
    that end inside a key tile, more rows than a row tile."""
    run_check(Problem([1, 300, 77, 530, 129], [1, 30, 0, 5, 129], d_c=d_c, d_r=d_r, page=page,
                      seed=d_c + page))


@pytest.mark.parametrize("page", [8, 24, 32, 48, 96, 120, 128, 200, 256, 1560])
def test_page_sizes(page):
    run_check(Problem([500, 3, 1700], [3, 2, 40], page=page, heads=5), 1, tokens=9)


@pytest.mark.parametrize("heads", [1, 3, 16, 40, 128, 200])
@pytest.mark.parametrize("new", [1, 2, 17])
def test_head_counts(heads, new):
    run_check(Problem([260, 40], [new, new], heads=heads, page=32))


@pytest.mark.parametrize("block", [0, 1, 2, 7, 64, 100, 1 << 30])
def test_masks(block):
    """No mask, token by token, blocks that end inside tiles and before the
    newest token's block does."""
    run_check(Problem([333, 200, 64, 1], [150, 200, 64, 1], heads=4, page=16), block)


@pytest.mark.parametrize("lens", [1, 2, 63, 64, 65, 127, 128, 129, 255, 256, 257, 383, 385])
def test_length_edges(lens):
    run_check(Problem([lens], [1], heads=12))
    run_check(Problem([lens], [lens], heads=3), 1)


def test_rows_that_see_nothing():
    """More new tokens than the stream holds: the first of them have negative
    places and see no key; an empty stream's rows are 0 too."""
    run_check(Problem([3, 0, 130, 0], [9, 4, 140, 0], heads=12, page=16), 1)
    run_check(Problem([0, 0], [1, 2], heads=12, page=16), 0)
    run_check(Problem([4], [300], heads=12, page=16), 3)


@pytest.mark.parametrize("lens,new", [([5000], [1]), ([40000], [2]), ([3000] * 7, [1] * 7),
                                      ([9001, 70, 1, 20011], [1, 1, 1, 3]),
                                      ([9001, 70, 1, 20011], [1, 70, 1, 300])])
def test_long_streams(lens, new):
    """Few rows and many keys: work split along the keys and joined."""
    p = Problem(lens, new, seed=9)
    o = run_check(p, 1, tokens=4)
    assert torch.equal(o, p.run(1))                   # and the same again, bit for bit


@pytest.mark.parametrize("d_c,d_r", [(512, 64), (256, 64), (64, 32)])
def test_long_streams_other_widths(d_c, d_r):
    run_check(Problem([7003, 100, 2500], [2, 90, 40], d_c=d_c, d_r=d_r, heads=16), 1, tokens=4)


@pytest.mark.parametrize("gain", [8.0, 40.0])
@pytest.mark.parametrize("new", [2, 60])
def test_sharp_scores(gain, new):
    """Scores up to hundreds: the running maximum keeps growing from tile to
    tile and partial results of different maxima are joined. A score's fp32
    error grows with its size, 224 * 2^-24 * |q||k| / sqrt(128) < 2^-9 here at
    gain 8; at gain 40 only finiteness and the winner's value are checked."""
    p = Problem([4000], [new], heads=4, gain=gain, seed=4)
    o = p.run(1)
    if gain == 8.0:
        p.check(o, 1, tokens=5)
        return
    assert torch.isfinite(o).all()
    c, kr = p.keys(0)
    q_c, q_r = p.q_c[0].double().cpu().numpy(), p.q_r[0].double().cpu().numpy()
    k = 4000 - new + 1
    x = (q_c @ c[:k].T + q_r @ kr[:k].T) / math.sqrt(128)
    for h in range(4):
        top = np.sort(x[h])[::-1]
        if top[0] - top[1] > 12:                      # the others weigh less than 2^-8 / 4000
            ref = c[np.argmax(x[h])]
            assert np.abs(o[0, h].double().cpu().numpy() - ref).max() <= 2.0 ** -6


def test_score_ramps():
    """Keys whose scores rise or fall steadily along the stream, so that the
    maximum moves in every tile or only in the first."""
    for sign in (1.0, -1.0):
        p = Problem([1500], [3], heads=2, seed=2)
        a = torch.arange(1500)
        ids = p.cache.table[0].cpu()[a // 64].long()
        p.cache.kr[0, ids, a % 64] = 0
        p.cache.kr[0, ids, a % 64, 0] = (sign * a / 12.5).to(torch.bfloat16).cuda()
        p.q_c.zero_()
        p.q_r.zero_()
        p.q_r[:, :, 0] = 4.0
        run_check(p, 1)


def test_layers_and_offsets_past_4_gib():
    """The last of two layers, 2.4 GiB each, pages far apart in it."""
    p = Problem([1], [1])
    cache = V.PagedCache.empty(2, 200000, 32, 2, 40, 192, 32)
    g = torch.Generator().manual_seed(1)
    p.lens, p.new = [1000, 33], [3, 1]
    ids = torch.randperm(200000, generator=g)[:34]
    ids[0] = 199999
    cache.table[0, :32] = ids[:32].to(torch.int32).cuda()
    cache.table[1, :2] = ids[32:].to(torch.int32).cuda()
    cache.lens.copy_(torch.tensor(p.lens))
    cache.c[1, ids] = torch.randn(34, 32, 192, generator=g).to(torch.bfloat16).cuda()
    cache.kr[1, ids] = torch.randn(34, 32, 32, generator=g).to(torch.bfloat16).cuda()
    p.cache, p.layer = cache, 1
    p.q_c = torch.randn(4, 12, 192, generator=g).to(torch.bfloat16).cuda()
    p.q_r = torch.randn(4, 12, 32, generator=g).to(torch.bfloat16).cuda()
    p.q_start = torch.tensor([0, 3, 4], dtype=torch.int32, device="cuda")
    p.keys = lambda s: tuple(
        t[1][cache.table[s].long()[torch.arange(p.lens[s], device="cuda") // 32],
             torch.arange(p.lens[s], device="cuda") % 32].double().cpu().numpy()
        for t in (cache.c, cache.kr))
    p.check(p.run(1), 1)


def test_many_streams():
    """More streams than a block has threads, of every small length."""
    rng = np.random.default_rng(3)
    lens = rng.integers(0, 90, 700)
    new = np.minimum(lens, rng.integers(0, 3, 700))
    run_check(Problem(lens.tolist(), new.tolist(), heads=2, page=16))


def test_other_stream_and_graph():
    p = Problem([900, 40], [2, 1])
    ref = p.run(1)
    s = torch.cuda.Stream()
    assert torch.equal(p.run(1, stream=s), ref)
    o = torch.full_like(ref, float("nan"))
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        V.mla_paged_attention(p.cache, 0, p.q_c, p.q_r, p.q_start, 128, 1, p.workspace, o)
    for _ in range(3):                                # lengths are read when it runs
        g.replay()
        torch.cuda.synchronize()
        assert torch.equal(o, ref)
        o.fill_(float("nan"))
    p.cache.lens[0] = 800
    p.lens[0] = 800
    g.replay()
    torch.cuda.synchronize()
    p.check(o, 1)


def test_dirty_workspace():
    p = Problem([30000, 500], [1, 3])
    ref = p.run(1)
    p.workspace.fill_(255)
    assert torch.equal(p.run(1), ref)
    p.workspace.fill_(127)
    assert torch.equal(p.run(1), ref)


def test_bad_metadata_is_recorded():
    p = Problem([300, 200], [2, 3])
    ref = p.run(1)

    def status():
        return V.mla_device_status(clear=True)

    q = p.q_start.clone()
    p.q_start[1], p.q_start[2] = 2, 6                 # past the tokens given
    o = p.run(1)
    assert status() == V.MLA_ERR_RANGE and torch.equal(o[:2], ref[:2])
    p.q_start[1], p.q_start[2] = 5, 2                 # not ascending
    p.run(1)
    assert status() == V.MLA_ERR_RANGE
    p.q_start.copy_(q)
    p.cache.lens[0] = 64 * p.max_pages + 1            # more than the table can name
    o = p.run(1)
    assert status() == V.MLA_ERR_RANGE and torch.equal(o[2:], ref[2:])
    p.cache.lens[0] = 300
    for bad in (-1, 10 ** 6, -2 ** 31):
        keep = p.cache.table[0, 1].item()
        p.cache.table[0, 1] = bad
        o = p.run(1)
        assert status() == V.MLA_ERR_RANGE
        assert torch.isfinite(o).all() and torch.equal(o[2:], ref[2:])
        p.cache.table[0, 1] = keep
    assert torch.equal(p.run(1), ref) and status() == V.MLA_OK


def test_refusals():
    p = Problem([30], [2])
    o = torch.empty_like(p.q_c)

    def call(**kw):
        a = dict(cache=p.cache, layer=0, q_c=p.q_c, q_r=p.q_r, q_start=p.q_start, head_dim=128,
                 causal_block=1, workspace=p.workspace, o=o)
        a.update(kw)
        V.mla_paged_attention(**a)

    for kw in (dict(layer=1), dict(layer=-1), dict(head_dim=0), dict(causal_block=-1),
               dict(workspace=p.workspace[:1])):
        with pytest.raises(V.MlaError) as e:
            call(**kw)
        assert e.value.code == V.MLA_ERR_ARG
    with pytest.raises(TypeError):
        call(q_c=p.q_c.float())
    with pytest.raises(ValueError):
        call(q_r=p.q_r[:1])
    with pytest.raises(ValueError):
        call(q_c=p.q_c.transpose(0, 1))
    with pytest.raises(ValueError):
        call(q_start=p.q_start[:1])
    with pytest.raises(TypeError):
        call(o=o.cpu())
    odd = V.PagedCache.empty(1, 4, 16, 1, 4, 96, 32)
    assert V.mla_paged_workspace_bytes(odd) == 0
    q = torch.zeros(1, 1, 96, dtype=torch.bfloat16, device="cuda")
    with pytest.raises(V.MlaError) as e:
        call(cache=odd, q_c=q, q_r=p.q_r[:1, :1].contiguous(), o=torch.empty_like(q),
             q_start=torch.tensor([0, 1], dtype=torch.int32, device="cuda"))
    assert e.value.code == V.MLA_ERR_UNSUPPORTED
    call(q_c=p.q_c[:0], q_r=p.q_r[:0], o=o[:0])


# ---------------------------------------------- streams of up to 16 rows on average
@pytest.mark.parametrize("page", [8, 9, 15, 16, 24, 32, 48, 64, 96, 100, 128, 200, 1560])
@pytest.mark.parametrize("d_c,d_r", [(192, 32), (64, 64)])
def test_one_token_page_sizes(page, d_c, d_r):
    run_check(Problem([1, 15, 16, 17, 129, 700, 3000], [1] * 7, page=page, d_c=d_c, d_r=d_r,
                      heads=8, seed=page), 1)


@pytest.mark.parametrize("d_c", [64, 128, 192, 256, 512])
@pytest.mark.parametrize("d_r", [32, 64])
@pytest.mark.parametrize("heads", [1, 5, 16])
def test_one_token_widths(d_c, d_r, heads):
    run_check(Problem([1000, 128, 0, 333], [1, 1, 0, 1], page=32, d_c=d_c, d_r=d_r, heads=heads),
              0)


@pytest.mark.parametrize("block", [0, 1, 3])
def test_mostly_idle_streams(block):
    """Few rows on average, and one stream with several tiles of 16 of them, more
    new tokens than another one holds."""
    new = [0] * 30
    new[3], new[17], new[29] = 21, 5, 1
    lens = [40] * 30
    lens[3], lens[17], lens[29] = 800, 3, 260
    run_check(Problem(lens, new, heads=12, page=16), block)


def test_one_token_sharp_and_long():
    p = Problem([20000, 64, 4097], [1, 1, 1], heads=16, gain=8.0, page=16, seed=11)
    o = run_check(p, 1)
    assert torch.equal(o, p.run(1))
    p.workspace.fill_(255)
    assert torch.equal(o, p.run(1))


def test_one_token_bad_pages_count_as_zeros():
    p = Problem([300, 200], [1, 1])
    ref = p.run(1)
    for bad in (-1, 10 ** 6, -2 ** 31):
        keep = p.cache.table[0, 1].item()
        p.cache.table[0, 1] = bad
        o = p.run(1)
        assert V.mla_device_status(clear=True) == V.MLA_ERR_RANGE
        assert torch.isfinite(o).all() and torch.equal(o[1], ref[1])
        p.cache.table[0, 1] = keep
    assert torch.equal(p.run(1), ref)


# At d_c = 512 two CTAs score 256 columns of c each (one of them k too) and add up what
# they send one another.

@pytest.mark.parametrize("part", ["first", "second", "k", "cancel"])
@pytest.mark.parametrize("d_r", [32, 64])
def test_wide_scores_from_either_half(part, d_r):
    """Scores that come from one CTA's columns alone, or cancel between the two."""
    p = Problem([700, 130, 65], [9, 1, 65], heads=3, d_c=512, d_r=d_r, page=32, seed=5, gain=6.0)
    q_c, q_r = p.q_c, p.q_r
    if part != "first":
        q_c[..., :256] = 0
    if part not in ("second", "cancel"):
        q_c[..., 256:] = 0
    if part != "k":
        q_r.zero_()
    if part == "cancel":
        q_c[..., :256] = -q_c[..., 256:]
        p.cache.c[..., 256:] = p.cache.c[..., :256]
    run_check(p, 1, tokens=9)


@pytest.mark.parametrize("rows", [1, 31, 32, 33, 80, 96, 97, 128, 129, 300])
@pytest.mark.parametrize("lens", [63, 64, 65, 200])
def test_wide_row_counts(rows, lens):
    """Warps without a row send nothing; tiles of one block and of several."""
    n = min(rows, lens)
    p = Problem([lens, lens + 1], [n, 1], heads=1 if rows <= lens else 5, d_c=512, d_r=64,
                page=16, seed=rows)
    run_check(p, 1, tokens=8)


def test_wide_many_blocks_same_bits():
    """Both exchange buffers many times over, and the same bits from call to call."""
    p = Problem([30000, 9000, 1, 17000], [3, 40, 1, 2], heads=16, d_c=512, d_r=64, seed=3)
    o = run_check(p, 1, tokens=3)
    for _ in range(5):
        assert torch.equal(p.run(), o)
