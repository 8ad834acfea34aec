"""Arrays that a window's calls write while they read others must not share memory with them:
refused before any pointer is used (no GPU needed)."""

import ctypes

import pytest

from paper_2605_30351_gb300 import videomla as V

STEP = 1 << 16
NAMES = ("c", "kr", "table", "lens", "refs", "plan", "dropped", "keep", "q_start", "pos", "pos_sink", "rows",
         "src", "dst")
AT = {n: (i + 16) * STEP for i, n in enumerate(NAMES)}
SEQS, PAGES, LIST, TOTAL = 3, 64, 8, 4
# bytes of each array that a call reads or writes
SIZE = dict(table=SEQS * LIST * 4, lens=SEQS * 4, refs=PAGES * 4, dropped=SEQS * 4, keep=SEQS * 4,
            q_start=SEQS * 4 + 4, pos=TOTAL * 12, pos_sink=TOTAL * 12, rows=TOTAL * 4, src=8, dst=8)


def call(name, **moved):
    at = dict(AT)
    at.update(moved)
    c = V.mla_paged_cache(layers=2, pages=PAGES, page_tokens=16, seqs=SEQS, max_pages=LIST, d_c=192, d_r=32,
                          **{n: at[n] for n in NAMES[:6]})
    w = V.mla_paged_window(window=5, sinks=1, dropped=at["dropped"])
    args = {"mla_pages_slide": (at["keep"], None),
            "mla_pages_window_fork": (at["src"], at["dst"], 2, None),
            "mla_paged_window_positions": (at["q_start"], TOTAL, 1, 64, 8, 3, at["pos"], at["pos_sink"],
                                           at["rows"], None)}[name]
    return getattr(V.load(), name)(ctypes.byref(c), ctypes.byref(w), *args)


def refused(name, a, b):
    """a moved to where it shares its first or its last word with b; a word further on either
    side nothing is wrong with the addresses, and the call goes on to look them up."""
    for at in (AT[b] - SIZE[a] + 4, AT[b] + SIZE[b] - 4, AT[b]):
        if a in ("table", "lens", "refs"):
            at = at // 16 * 16 if at > AT[b] else -(-at // 16) * 16  # the cache's own are aligned
        assert call(name, **{a: at}) == V.MLA_ERR_ARG, (name, a, b, at - AT[b])
    if V.torch.cuda.is_available():                   # these are no addresses of a GPU's
        return
    for at in (AT[b] - SIZE[a] - 12, AT[b] + SIZE[b] + 12):
        if at % 16 == 0 or a not in ("table", "lens", "refs"):
            assert call(name, **{a: at}) == V.MLA_ERR_CUDA, (name, a, b)


@pytest.mark.parametrize("a,b", [(a, b) for a in ("dropped", "keep") for b in ("table", "lens", "refs")] +
                         [("keep", "dropped"), ("lens", "table"), ("refs", "table"), ("lens", "refs")])
def test_slide(a, b):
    """It writes table, lens, refs and dropped, a block per stream, while others read them and
    keep."""
    refused("mla_pages_slide", a, b)


@pytest.mark.parametrize("a", ["pos", "pos_sink", "rows"])
def test_positions_and_the_page_table(a):
    """Pages are looked up while other blocks write pos, pos_sink and rows."""
    refused("mla_paged_window_positions", a, "table")


@pytest.mark.parametrize("a,b", [(a, b) for a in ("dropped", "src", "dst") for b in ("table", "lens", "refs")] +
                         [("src", "dropped"), ("dst", "dropped")])
def test_branches(a, b):
    """They write the new stream's row of the table, its length and count, and the pages'
    reference counts."""
    refused("mla_pages_window_fork", a, b)
