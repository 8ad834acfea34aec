"""Page operations and the paged append on the GPU against the oracle's rules:
metadata equal integer for integer, contents bit for bit (the rotated keys
within one rounding)."""

import numpy as np
import pytest
import torch

from oracle import paged_oracle as O
from paper_2605_30351_gb300 import videomla as V

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    V.load()
    V.mla_device_status(clear=True)
    yield
    assert V.mla_device_status(clear=True) == V.MLA_OK


def i32(v):
    return torch.tensor(np.asarray(v), dtype=torch.int32, device="cuda")


def both(layers=2, pages=40, tokens=8, seqs=6, max_pages=12, d_c=64, d_r=32, seed=0):
    """An empty pool on both sides whose rows hold the same garbage."""
    cache = V.PagedCache.empty(layers, pages, tokens, seqs, max_pages, d_c, d_r)
    g = torch.Generator().manual_seed(seed)
    for t in (cache.c, cache.kr):
        t.copy_(torch.randn(t.shape, generator=g).to(torch.bfloat16))
    o = O.Pages(layers, pages, tokens, seqs, max_pages, d_c, d_r)
    o.c, o.kr = cache.c.double().cpu().numpy(), cache.kr.double().cpu().numpy()
    return cache, o


def same(cache, o, contents=True):
    assert np.array_equal(cache.table.cpu().numpy(), o.table)
    assert np.array_equal(cache.lens.cpu().numpy(), o.lens)
    assert np.array_equal(cache.refs.cpu().numpy(), o.refs)
    if contents:
        for t, ref in ((cache.c, o.c), (cache.kr, o.kr)):
            assert np.array_equal(t.double().cpu().numpy(), ref)


@pytest.mark.parametrize("seed,tokens,seqs", [(1, 8, 6), (2, 16, 3), (3, 24, 11), (4, 8, 40)])
def test_random_operations(seed, tokens, seqs):
    """Grow, shrink, free, branch, pack and copy in random order, several
    streams in one call, the pool running out now and then."""
    cache, o = both(tokens=tokens, seqs=seqs, pages=61, seed=seed)
    rng = np.random.default_rng(seed)
    cap = 12 * tokens
    for step in range(60):
        kind = rng.integers(6)
        if kind <= 2:
            new = np.where(rng.random(seqs) < 0.5, rng.integers(0, cap + 1, seqs), -1)
            if kind == 1:                             # mostly growth by a little
                new = np.minimum(cap, o.lens + rng.integers(0, 2 * tokens, seqs))
            cache_new = i32(new)
            V.mla_pages_resize(cache, cache_new)
            o.resize(new)
        elif kind == 3:
            empty = [s for s in range(seqs) if o.lens[s] == 0]
            full = [s for s in range(seqs) if o.lens[s] > 0]
            if empty and full:
                src = rng.choice(full, len(empty))
                V.mla_pages_fork(cache, i32(src), i32(empty))
                o.fork(src, empty)
        elif kind == 4:
            V.mla_pages_compact(cache, cache.table, cache.refs)
            o.compact()
        else:
            pg = rng.permutation(61)
            V.mla_pages_copy(cache, i32(pg[:9]), i32(pg[9:18]))
            o.c[:, pg[9:18]], o.kr[:, pg[9:18]] = o.c[:, pg[:9]], o.kr[:, pg[:9]]
        same(cache, o, contents=step % 4 == 3)
        status = V.mla_device_status(clear=True)
        assert status == (V.MLA_ERR_RANGE if o.range_error else V.MLA_OK), step
        o.range_error = False
    same(cache, o)


@pytest.mark.parametrize("pages", [1, 5, 1024, 1025, 5000, 70000])
def test_compact_into_other_buffers(pages):
    """Packing with new metadata buffers leaves the old ones as they were; pool
    sizes around the block and grid sizes, none, some and all pages in use."""
    for fill in (0.0, 0.4, 1.0):
        cache, o = both(layers=1, pages=pages, tokens=8, seqs=3, max_pages=pages, d_c=8, d_r=8)
        rng = np.random.default_rng(pages)
        live = np.flatnonzero(rng.random(pages) < fill)
        rng.shuffle(live)
        cut = len(live) // 2
        o.table[0, :cut], o.table[1, :len(live) - cut] = live[:cut], live[cut:]
        o.table[2, :cut] = live[:cut]
        o.lens[:] = [8 * cut, 8 * (len(live) - cut), 8 * cut]
        o.refs[live[:cut]], o.refs[live[cut:]] = 2, 1
        for t, ref in ((cache.table, o.table), (cache.lens, o.lens), (cache.refs, o.refs)):
            t.copy_(torch.from_numpy(ref))
        before = cache.table.clone(), cache.refs.clone()
        table, refs = torch.empty_like(cache.table), torch.empty_like(cache.refs)
        V.mla_pages_compact(cache, table, refs)
        assert torch.equal(cache.table, before[0]) and torch.equal(cache.refs, before[1])
        c0 = cache.c.clone()
        V.mla_pages_compact(cache, table, refs)       # the same again: nothing changes
        assert torch.equal(cache.c, c0)
        cache.table.copy_(table)
        cache.refs.copy_(refs)
        if pages <= 5000:                             # the oracle walks page by page
            o.compact()
            same(cache, o)
        else:
            n = len(live)
            assert (refs[:n] > 0).all() and (refs[n:] == 0).all()
            at = cache.table[0, :cut].long()
            old = torch.from_numpy(o.c)[0, live[:cut]]
            assert torch.equal(cache.c[0, at].double().cpu(), old)


def test_branches_do_not_see_each_other():
    """Three streams share a partly filled page; two of them grow in one call,
    then the third: each gets rows of its own, and the page itself is free."""
    cache, o = both(seqs=4, tokens=16)
    for op in (lambda: (V.mla_pages_resize(cache, i32([20, -1, -1, -1])),
                        o.resize([20, -1, -1, -1])),
               lambda: (V.mla_pages_fork(cache, i32([0, 0]), i32([1, 2])), o.fork([0, 0], [1, 2])),
               lambda: (V.mla_pages_resize(cache, i32([-1, 21, 40, -1])),
                        o.resize([-1, 21, 40, -1])),
               lambda: (V.mla_pages_resize(cache, i32([33, -1, -1, 0])), o.resize([33, -1, -1, 0]))):
        op()
        same(cache, o)
    assert len(set(o.table[:3, 1])) == 3 and len(set(o.table[:3, 0])) == 1


def test_bad_requests_are_recorded_and_skipped():
    cache, o = both(seqs=4, tokens=8, pages=10, max_pages=8)
    V.mla_pages_resize(cache, i32([24, 9, -1, 0]))
    o.resize([24, 9, -1, 0])
    for src, dst in (([0], [1]), ([0], [4]), ([-1], [2]), ([0], [0])):
        V.mla_pages_fork(cache, i32(src), i32(dst))
        assert V.mla_device_status(clear=True) == V.MLA_ERR_RANGE
        same(cache, o)
    V.mla_pages_resize(cache, i32([65, -1, 8, -1]))   # 65 tokens: past max_pages
    o.resize([65, -1, 8, -1])
    assert V.mla_device_status(clear=True) == V.MLA_ERR_RANGE
    same(cache, o)
    V.mla_pages_resize(cache, i32([64, 16, 64, 1]))   # the pool holds the first of them
    o.resize([64, 16, 64, 1])
    assert V.mla_device_status(clear=True) == V.MLA_ERR_RANGE
    same(cache, o)
    V.mla_pages_copy(cache, i32([0, 10]), i32([9, 1]))
    o.c[:, 9], o.kr[:, 9] = o.c[:, 0], o.kr[:, 0]
    assert V.mla_device_status(clear=True) == V.MLA_ERR_RANGE
    same(cache, o)
    V.mla_pages_resize(cache, i32([2 ** 31 - 1] * 4))
    assert V.mla_device_status(clear=True) == V.MLA_ERR_RANGE
    same(cache, o)


def test_many_streams():
    """More streams than the metadata kernel has threads."""
    cache, o = both(layers=1, seqs=2500, tokens=8, pages=6000, max_pages=4, d_c=8, d_r=8)
    rng = np.random.default_rng(7)
    for _ in range(4):
        new = rng.integers(-1, 33, 2500)
        V.mla_pages_resize(cache, i32(new))
        o.resize(new)
        same(cache, o)
        V.mla_device_status(clear=True)


# -------------------------------------------------------------------- append
@pytest.mark.parametrize("d_c,d_r,half,axes", [(192, 32, False, 3), (512, 64, False, 1),
                                               (64, 64, True, 1), (8, 8, False, 3)])
@pytest.mark.parametrize("seqs", [1, 5, 33, 100])
def test_append(d_c, d_r, half, axes, seqs):
    rng = np.random.default_rng(seqs + d_c)
    tokens = 8 if seqs > 5 else 24
    cache, o = both(tokens=tokens, seqs=seqs, pages=12 * seqs + 3, d_c=d_c, d_r=d_r)
    lens = rng.integers(0, 12 * tokens + 1, seqs)
    V.mla_pages_resize(cache, i32(lens))
    o.resize(lens)
    n = np.minimum(lens, np.where(rng.random(seqs) < 0.3, 0, rng.integers(0, 60, seqs)))
    q = np.concatenate([[0], np.cumsum(n)])
    total = int(q[-1])
    pairs = (d_r // 2 - 2 * (d_r // 6), d_r // 6, d_r // 6) if axes == 3 else (d_r // 2, 0, 0)
    tab = V.mla_rope_scaled_table_fill(d_r, 100)
    rope = V.Rope(torch.from_numpy(tab).cuda(), pairs, half=half, axes=axes)
    g = torch.Generator().manual_seed(1)
    c_new = torch.randn(total, d_c, generator=g).to(torch.bfloat16)
    kr_new = torch.randn(total, d_r, generator=g).to(torch.bfloat16)
    pos = torch.randint(0, 100, (total, axes), generator=g, dtype=torch.int32)
    V.mla_paged_append(cache, 1, c_new.cuda(), kr_new.cuda(), i32(q), pos.cuda(), rope)
    rot = O.rotate(kr_new.double().numpy()[:, None], pos.numpy(), tab, pairs, 0, half)[:, 0]
    o.append(1, c_new.double().numpy(), rot, q)
    assert np.array_equal(cache.c.double().cpu().numpy(), o.c)
    # one rounding to bf16 of fp32 arithmetic on values up to about 4
    err = np.abs(cache.kr.double().cpu().numpy() - o.kr)
    assert (err <= 2.0 ** -8 * np.abs(o.kr) + 2.0 ** -20).all()
    same(cache, o, contents=False)


def test_append_rejects_places_without_a_page():
    cache, o = both(seqs=2, tokens=8)
    V.mla_pages_resize(cache, i32([12, 4]))
    o.resize([12, 4])
    tab = V.mla_rope_scaled_table_fill(32, 4)
    rope = V.Rope(torch.from_numpy(tab).cuda(), (16, 0, 0))
    c = torch.ones(6, 64, dtype=torch.bfloat16, device="cuda")
    k = torch.ones(6, 32, dtype=torch.bfloat16, device="cuda")
    zero = torch.zeros(6, 1, dtype=torch.int32, device="cuda")

    def call(q, pos=zero):
        V.mla_paged_append(cache, 0, c, k, i32(q), pos, rope)
        return V.mla_device_status(clear=True)

    before = cache.c.clone()
    assert call([0, 1, 7]) == V.MLA_ERR_RANGE         # q_start past the tokens given
    assert torch.equal(cache.c[:, o.table[1, 0]], before[:, o.table[1, 0]])
    assert call([0, 0, 6]) == V.MLA_ERR_RANGE         # 6 new tokens of a stream of 4
    assert call([0, 6, 6], zero + 4) == V.MLA_ERR_RANGE   # positions past the table
    assert call([0, 4, 6]) == V.MLA_OK
    V.mla_paged_append(cache, 0, c[:0], k[:0], i32([0, 0, 0]), zero[:0], rope)


def test_append_past_4_gib():
    """Rows of the last layer of a pool whose byte offsets pass 32 bits."""
    cache = V.PagedCache.empty(2, 200000, 32, 1, 4, 192, 32)      # 2.4 GiB a layer
    cache.table.copy_(i32([[199999, 3, 150000, -1]]))
    cache.lens.fill_(90)
    cache.refs[[199999, 3, 150000]] = 1
    tab = V.mla_rope_scaled_table_fill(32, 100)
    rope = V.Rope(torch.from_numpy(tab).cuda(), (16, 0, 0))
    g = torch.Generator().manual_seed(3)
    c = torch.randn(90, 192, generator=g).to(torch.bfloat16).cuda()
    k = torch.randn(90, 32, generator=g).to(torch.bfloat16).cuda()
    zero = torch.zeros(90, 1, dtype=torch.int32, device="cuda")
    V.mla_paged_append(cache, 1, c, k, i32([0, 90]), zero, rope)
    at = torch.tensor([199999] * 32 + [3] * 32 + [150000] * 26)
    row = torch.arange(90) % 32
    assert torch.equal(cache.c[1, at, row], c) and torch.equal(cache.kr[1, at, row], k)
    assert cache.c[0].abs().max() == 0
    V.mla_pages_copy(cache, i32([199999]), i32([0]))
    assert torch.equal(cache.c[1, 0], c[:32])


def test_refusals():
    cache, _ = both(seqs=4)
    with pytest.raises(ValueError):
        V.mla_pages_resize(cache, i32([1, 2, 3]))
    with pytest.raises(TypeError):
        V.mla_pages_resize(cache, torch.zeros(4, dtype=torch.int64, device="cuda"))
    with pytest.raises(ValueError):
        V.mla_pages_fork(cache, i32([0, 1]), i32([2]))
    with pytest.raises(V.MlaError):
        V.mla_pages_fork(cache, i32([0] * 5), i32([1] * 5))
    with pytest.raises(V.MlaError):
        V.PagedCache.empty(1, 4, 4, 1, 1, 64, 32)     # pages of fewer than 8 tokens
    with pytest.raises(TypeError):
        V.PagedCache(cache.c.cpu(), cache.kr, cache.table, cache.lens, cache.refs)
