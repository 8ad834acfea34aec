"""Host side of the operators of streams whose window slides, no GPU needed: argument
rules, all of them checked before any pointer is used, and how their kernels read."""

import ctypes
import os
import re

import numpy as np
import pytest

from oracle import paged_oracle as O
from paper_2605_30351_gb300 import videomla as V

FAKE = 1 << 20
CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))),
                    "paper_2605_30351_gb300", "csrc")


def paged(**kw):
    a = dict(c=FAKE, kr=FAKE, table=FAKE, lens=FAKE, refs=FAKE, plan=FAKE, layers=2, pages=64,
             page_tokens=16, seqs=3, max_pages=8, d_c=192, d_r=32)
    a.update(kw)
    return V.mla_paged_cache(**a)


ARGS = {
    "mla_paged_window_attention": dict(
        layer=0, q_c=FAKE, q_r=FAKE, q_r_sink=FAKE, total=4, heads=12, q_start=FAKE, head_dim=128,
        block=1, workspace=FAKE, nbytes=1 << 30, o=FAKE, stream=None),
    "mla_paged_window_plan": dict(n_new=FAKE + (1 << 16), q_start=FAKE + (2 << 16),
                                  new_lens=FAKE + (3 << 16), stream=None),
    "mla_paged_window_positions": dict(
        q_start=FAKE + (1 << 16), total=4, block=1, frame=64, width=8, axes=3, pos=FAKE + (2 << 16),
        pos_sink=FAKE + (3 << 16), rows=FAKE + (4 << 16), stream=None),
    "mla_pages_slide": dict(keep=FAKE, stream=None),
    "mla_pages_window_fork": dict(src=FAKE, dst=FAKE, n=1, stream=None),
}


def call(name, cache=None, window=5, sinks=1, dropped=FAKE + (9 << 16), null=False, **kw):
    a = dict(ARGS[name])
    assert set(kw) <= set(a)
    a.update(kw)
    c = paged() if cache is None else cache
    w = V.mla_paged_window(window=window, sinks=sinks, dropped=dropped)
    return getattr(V.load(), name)(ctypes.byref(c), None if null else ctypes.byref(w), *a.values())


@pytest.mark.parametrize("name", ARGS)
def test_the_window_and_the_cache_are_checked(name):
    for bad in (dict(window=0), dict(window=-5), dict(sinks=-1), dict(dropped=FAKE + 2), dict(null=True),
                dict(cache=paged(c=None)), dict(cache=paged(kr=FAKE + 8)), dict(cache=paged(lens=FAKE + 4)),
                dict(cache=paged(seqs=0)), dict(cache=paged(page_tokens=7)), dict(cache=paged(refs=None))):
        assert call(name, **bad) == V.MLA_ERR_ARG, bad


def test_calls_that_write_it_need_dropped():
    assert call("mla_pages_slide", dropped=None) == V.MLA_ERR_ARG
    assert call("mla_pages_window_fork", dropped=None) == V.MLA_ERR_ARG


@pytest.mark.parametrize("name,bad", [
    *[("mla_paged_window_attention", b) for b in (
        dict(layer=2), dict(layer=-1), dict(total=-1), dict(heads=0), dict(head_dim=0), dict(block=-1),
        dict(total=1 << 20, heads=(1 << 10) + 1), dict(q_c=None), dict(q_r=None), dict(q_start=None),
        dict(workspace=None), dict(o=None), dict(q_c=FAKE + 8), dict(q_r=FAKE + 8), dict(q_r_sink=FAKE + 8),
        dict(q_start=FAKE + 2), dict(workspace=FAKE + 8), dict(o=FAKE + 8), dict(nbytes=0))],
    *[("mla_paged_window_plan", b) for b in (
        dict(n_new=None), dict(q_start=None), dict(new_lens=None), dict(n_new=FAKE + 1),
        dict(q_start=FAKE + 2), dict(new_lens=FAKE + 3))],
    *[("mla_paged_window_positions", b) for b in (
        dict(total=-1), dict(block=-1), dict(frame=0), dict(width=0), dict(width=65), dict(axes=2), dict(axes=0),
        dict(pos=None), dict(q_start=None), dict(pos=FAKE + 2), dict(pos_sink=FAKE + 2), dict(rows=FAKE + 1),
        dict(q_start=FAKE + 1))],
    *[("mla_pages_slide", b) for b in (dict(keep=None), dict(keep=FAKE + 2))],
    *[("mla_pages_window_fork", b) for b in (
        dict(n=-1), dict(n=4), dict(src=None), dict(dst=None), dict(src=FAKE + 2), dict(dst=FAKE + 2))],
])
def test_arguments_are_checked(name, bad):
    assert call(name, **bad) == V.MLA_ERR_ARG


def test_arrays_that_overlap_are_refused():
    """seqs = 3: n_new, new_lens, lens and dropped take 12 bytes, q_start 16."""
    at = ARGS["mla_paged_window_plan"]
    for bad in (dict(n_new=at["q_start"] + 12), dict(new_lens=at["n_new"] + 8),
                dict(q_start=at["new_lens"] - 12), dict(new_lens=FAKE), dict(q_start=FAKE + (9 << 16) + 8),
                dict(q_start=FAKE + 8)):
        assert call("mla_paged_window_plan", **bad) == V.MLA_ERR_ARG, bad
    at = ARGS["mla_paged_window_positions"]
    for bad in (dict(pos=at["pos_sink"] + 44), dict(pos_sink=at["rows"] - 44), dict(rows=at["q_start"] + 12),
                dict(pos=FAKE), dict(rows=FAKE + (9 << 16))):
        assert call("mla_paged_window_positions", **bad) == V.MLA_ERR_ARG, bad


def test_windows_past_32_bits_are_refused():
    for bad in ((1 << 32) + 5, 1 << 31):
        with pytest.raises(ValueError):
            V.PagedWindow(bad)
        with pytest.raises(ValueError):
            V.PagedWindow(5, bad)


def test_a_workspace_one_byte_short_is_refused():
    need = V.load().mla_paged_workspace_bytes(ctypes.byref(paged()))
    assert call("mla_paged_window_attention", nbytes=need - 1) == V.MLA_ERR_ARG


@pytest.mark.parametrize("d_c,d_r", [(96, 32), (384, 32), (192, 16), (192, 128)])
def test_widths_without_a_kernel(d_c, d_r):
    assert call("mla_paged_window_attention", cache=paged(d_c=d_c, d_r=d_r)) == V.MLA_ERR_UNSUPPORTED


@pytest.mark.parametrize("name", [f for f in sorted(os.listdir(CSRC)) if re.match(r"page", f)])
def test_inputs_are_read_coherently(name):
    """The kernels start while the stream's previous one, which may write what they read,
    still runs: none of their loads goes through the non-coherent path."""
    with open(os.path.join(CSRC, name)) as f:
        code = re.sub(r"//[^\n]*", "", f.read())
    assert not re.findall(r"__ldg|\.nc\b|__restrict__|__ldca", code)


def test_oracle_window_by_hand():
    """A stream of 10 tokens, page 4, 2 sinks: what its tokens see, before and after 4 were
    given back (places 4 .. 7 became 4 .. 5 of what is held, the rest follows)."""
    sees = O.window_sees(9, 10, 0, 1, 3, 2, 4)
    assert [v.tolist() for v in sees] == [[0, 1], [7, 8, 9]]
    assert [v.tolist() for v in O.window_sees(5, 6, 4, 1, 3, 2, 4)] == [[0, 1], [4, 5]]
    assert [v.tolist() for v in O.window_sees(0, 10, 0, 1, 3, 2, 4)] == [[0], []]
    assert [v.tolist() for v in O.window_sees(2, 10, 0, 1, 3, 2, 4)] == [[0, 1], [2]]
    assert [v.tolist() for v in O.window_sees(4, 10, 0, 5, 3, 0, 4)] == [[], [2, 3, 4]]
    assert [v.tolist() for v in O.window_sees(3, 10, 0, 0, 3, 0, 4)] == [[], [7, 8, 9]]
    assert [v.tolist() for v in O.window_sees(-1, 10, 0, 0, 3, 1, 4)] == [[], []]


@pytest.mark.parametrize("seed", range(5))
def test_oracle_of_a_slid_stream_is_that_of_the_whole_one(seed):
    """What slid streams compute is what the whole stream's tokens compute, as long as the
    window's tokens are kept."""
    rng = np.random.default_rng(seed)
    P, sinks, window, block = 8, int(rng.integers(0, 20)), int(rng.integers(1, 60)), int(rng.choice([1, 5]))
    total, new = 300, 4
    first = total - new
    keep = window + new - 1
    c, kr = rng.standard_normal((total, 6)), rng.standard_normal((total, 4))
    pages = O.Pages(1, 60, P, 1, 60, 6, 4)
    pages.resize([total])
    gone = np.zeros(1, np.int64)
    O.slide(pages, gone, [keep], sinks)
    back = int(gone[0])
    f = O.front(sinks, P)
    held = np.r_[0:f, f + back:total]
    assert len(held) == pages.lens[0] and back % P == 0 and total - f - back >= min(keep, total - f)
    for i in range(new):
        q = rng.standard_normal((2, 6)), rng.standard_normal((2, 4)), rng.standard_normal((2, 4))
        whole, _ = O.attend_window(*q, c, kr, O.window_sees(first + i, total, 0, block, window, sinks, P), 16)
        part, _ = O.attend_window(*q, c[held], kr[held],
                                  O.window_sees(len(held) - new + i, len(held), back, block, window, sinks, P), 16)
        assert np.abs(whole - part).max() <= 1e-12
