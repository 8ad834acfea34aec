"""Attention over the paged latent cache where its inputs lie at an edge of what the
entry point accepts."""

import numpy as np
import pytest
import torch

from oracle import paged_oracle as O
from paper_2605_30351_gb300 import videomla as V
from test_gpu_paged_attention import REL, Problem

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


# A key that is not finite, the last one of each stream: the newest token sees it, and
# alone in its block of 64 or 128 keys. Whether a share of the work begins with that
# block, ends before it or holds the whole tile depends on the sizes; the answer must
# not. What the earlier tokens get is left open.
LEN = 513
PLACES = [
    # streams, new tokens of each, heads
    (60, 4, 12),      # tiles of 48 rows, cut by two or three shares
    (60, 30, 12),     # two tiles and more a stream
    (400, 4, 12),     # most tiles whole
    (3, 4, 12),       # tiles cut by many shares
    (3, 2, 12),       # short tiles
    (60, 1, 12),      # tiles of 16 rows
    (3, 1, 12),
]


def with_key(where, value, streams, new, heads, d_c, seed=0):
    """A problem whose streams' last keys hold `value` in one column of c or k."""
    p = Problem([LEN] * streams, [new] * streams, heads=heads, d_c=d_c, page=64, seed=seed)
    last = p.cache.table[:, (LEN - 1) // 64].long()
    t = p.cache.c if where == "c" else p.cache.kr
    t[p.layer, last, (LEN - 1) % 64, 5] = value
    return p


def newest(p):
    """(stream, its newest token's row)."""
    return list(enumerate(np.cumsum(p.new) - 1))


def host(*tensors):
    return (t.double().cpu().numpy() for t in tensors)


@pytest.mark.parametrize("d_c", [64, 128, 192, 256, 512])
@pytest.mark.parametrize("streams,new,heads", PLACES)
@pytest.mark.parametrize("where", ["c", "k"])
def test_nan_in_a_visible_key(where, streams, new, heads, d_c):
    """Its score is NaN, so every weight and every value of the rows is."""
    p = with_key(where, float("nan"), streams, new, heads, d_c)
    o = p.run(1)
    bad = [s for s, i in newest(p) if not torch.isnan(o[i]).all()]
    assert not bad, bad


@pytest.mark.parametrize("d_c", [64, 128, 192, 256, 512])
@pytest.mark.parametrize("streams,new,heads", PLACES)
@pytest.mark.parametrize("where", ["c", "k"])
def test_infinity_in_a_visible_key(where, streams, new, heads, d_c):
    """Where the query's value there is positive, the score is inf and all weights are
    inf - inf: NaN. Where it is negative the score is -inf and the weight 0: the row is
    that of the other keys (the tolerance of test_gpu_paged_attention), but for the
    column of c that holds the infinity, 0 * inf."""
    p = with_key(where, float("inf"), streams, new, heads, d_c, seed=1)
    o, q_c, q_r, table, c_all, kr_all = host(p.run(1), p.q_c, p.q_r, p.cache.table,
                                             p.cache.c[p.layer], p.cache.kr[p.layer])
    a = np.arange(LEN - 1)
    for s, i in newest(p):
        q = (q_c if where == "c" else q_r)[i, :, 5]
        assert (q != 0).all()
        at = table[s].astype(int)[a // 64], a % 64
        args = q_c[i:i + 1], q_r[i:i + 1], c_all[at], kr_all[at], p.head_dim, 0
        ref, size = O.attend(*args)[0], O.attend(*args, np.abs(c_all[at]))[0]
        for h in range(heads):
            if q[h] > 0:
                assert np.isnan(o[i, h]).all(), (s, h)
                continue
            cols = np.arange(d_c) != 5 if where == "c" else np.ones(d_c, bool)
            assert np.isnan(o[i, h, ~cols]).all(), (s, h)
            assert (np.abs(o[i, h] - ref[h]) <= REL * size[h])[cols].all(), (s, h)


@pytest.mark.parametrize("streams,new,heads,d_c", [
    (97, 3, 12, 192),      # one stream more than threads that look for a share's end
    (300, 5, 4, 128),
    (1000, 2, 9, 64),
    (150, 1, 2, 512),
    (100, 90, 3, 192),     # two row tiles a stream: CTA pairs
])
def test_many_streams_in_tiles_of_128_rows(streams, new, heads, d_c):
    """More streams than the share search has threads; idle and empty ones among
    them. All of them against the oracle's attention."""
    rng = np.random.default_rng(streams)
    lens = rng.integers(new, 200, streams)
    n = np.where(np.arange(streams) % 7 == 3, 0, new)
    lens[5::50] = 0
    n[5::50] = 0
    p = Problem(lens.tolist(), n.tolist(), heads=heads, d_c=d_c, page=16, seed=streams)
    o, q_c, q_r, table, c_all, kr_all = host(p.run(1), p.q_c, p.q_r, p.cache.table,
                                             p.cache.c[p.layer], p.cache.kr[p.layer])
    end = np.cumsum(n)
    for s in np.flatnonzero(n):
        a = np.arange(lens[s])
        at = table[s].astype(int)[a // 16], a % 16
        i = slice(end[s] - n[s], end[s])
        args = q_c[i], q_r[i], c_all[at], kr_all[at], p.head_dim, 1
        ref, size = O.attend(*args), O.attend(*args, np.abs(c_all[at]))
        assert (np.abs(o[i] - ref) <= REL * size).all(), s
