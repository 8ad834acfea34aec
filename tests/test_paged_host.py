"""Host side of the rotary and paged-cache entry points, no GPU needed: struct
layouts, argument rules (checked before any pointer is used), the scaled RoPE
tables, and the oracle's own page rules."""

import ctypes

import numpy as np
import pytest

from oracle import paged_oracle as O
from paper_2605_30351_gb300 import videomla as V

FAKE = ctypes.c_void_p(1 << 20)
ODD = ctypes.c_void_p((1 << 20) + 2)


def paged(**kw):
    a = dict(c=FAKE, kr=FAKE, table=FAKE, lens=FAKE, refs=FAKE, plan=FAKE, layers=2, pages=64,
             page_tokens=16, seqs=3, max_pages=8, d_c=192, d_r=32)
    a.update(kw)
    return V.mla_paged_cache(**a)


def rope(**kw):
    a = dict(table=FAKE, table_len=128, pairs_t=6, pairs_h=5, pairs_w=5, axes=3, offset=0,
             layout=0)
    a.update(kw)
    return V.mla_rope(**a)


def test_struct_layouts():
    assert ctypes.sizeof(V.mla_rope) == 40 and V.mla_rope.layout.offset == 32
    assert ctypes.sizeof(V.mla_paged_cache) == 80 and V.mla_paged_cache.d_r.offset == 72


@pytest.mark.parametrize("bad", [
    dict(layers=0), dict(pages=0), dict(page_tokens=7), dict(seqs=0), dict(seqs=65537),
    dict(max_pages=0), dict(d_c=0), dict(d_c=100), dict(d_r=4), dict(d_r=36),
    dict(pages=1 << 27, page_tokens=16), dict(max_pages=1 << 27, page_tokens=16)])
def test_paged_sizes_are_checked(bad):
    lib = V.load()
    ok, c = paged(), paged(**bad)
    assert lib.mla_paged_check(ctypes.byref(ok)) == V.MLA_OK
    assert lib.mla_pages_plan_bytes(ctypes.byref(ok)) >= 4 * (2 + 3 * 64)
    assert lib.mla_paged_check(ctypes.byref(c)) == V.MLA_ERR_ARG
    assert lib.mla_pages_plan_bytes(ctypes.byref(c)) == 0
    for rc in (lib.mla_pages_resize(ctypes.byref(c), FAKE, None),
               lib.mla_pages_fork(ctypes.byref(c), FAKE, FAKE, 1, None),
               lib.mla_pages_copy(ctypes.byref(c), FAKE, FAKE, 1, None),
               lib.mla_pages_compact(ctypes.byref(c), FAKE, FAKE, None),
               lib.mla_paged_append(ctypes.byref(c), 0, FAKE, FAKE, 1, FAKE, FAKE,
                                    ctypes.byref(rope()), None)):
        assert rc == V.MLA_ERR_ARG
    assert lib.mla_paged_check(None) == V.MLA_ERR_ARG


def test_paged_pointers_are_checked():
    lib = V.load()
    for name in ("c", "kr", "table", "lens", "refs", "plan"):
        for p in (None, ODD):
            c = paged(**{name: p})
            assert lib.mla_pages_resize(ctypes.byref(c), FAKE, None) == V.MLA_ERR_ARG
    c = ctypes.byref(paged())
    assert lib.mla_pages_resize(c, None, None) == V.MLA_ERR_ARG
    assert lib.mla_pages_fork(c, None, FAKE, 1, None) == V.MLA_ERR_ARG
    assert lib.mla_pages_fork(c, FAKE, FAKE, -1, None) == V.MLA_ERR_ARG
    assert lib.mla_pages_copy(c, FAKE, None, 1, None) == V.MLA_ERR_ARG
    assert lib.mla_pages_compact(c, FAKE, None, None) == V.MLA_ERR_ARG
    r = ctypes.byref(rope())
    for args in ((2, FAKE, FAKE, 1, FAKE, FAKE, r), (-1, FAKE, FAKE, 1, FAKE, FAKE, r),
                 (0, None, FAKE, 1, FAKE, FAKE, r), (0, ODD, FAKE, 1, FAKE, FAKE, r),
                 (0, FAKE, FAKE, -1, FAKE, FAKE, r), (0, FAKE, FAKE, 1, None, FAKE, r),
                 (0, FAKE, FAKE, 1, FAKE, None, r), (0, FAKE, FAKE, 1, FAKE, FAKE, None),
                 (0, FAKE, FAKE, 1, FAKE, FAKE, ctypes.byref(rope(offset=2))),
                 (0, FAKE, FAKE, 1, FAKE, FAKE, ctypes.byref(rope(pairs_t=7)))):
        assert lib.mla_paged_append(c, *args, None) == V.MLA_ERR_ARG


@pytest.mark.parametrize("bad", [
    dict(table=None), dict(table=ctypes.c_void_p((1 << 20) + 4)), dict(table_len=0),
    dict(pairs_t=-1), dict(pairs_t=0, pairs_h=0, pairs_w=0), dict(axes=2), dict(axes=1),
    dict(offset=-2), dict(layout=2), dict(offset=97)])
def test_rope_arguments_are_checked(bad):
    lib = V.load()
    r = ctypes.byref(rope(**bad))
    assert lib.mla_rope_apply(r, FAKE, FAKE, FAKE, 0, 1, 1, 128, 128, 128, 128, 128, 0,
                              None) == V.MLA_ERR_ARG


def test_rope_apply_arguments():
    lib = V.load()
    r = ctypes.byref(rope())
    tail = (0, None)
    st = (128, 128, 128, 128)
    assert lib.mla_rope_apply(None, FAKE, FAKE, FAKE, 0, 1, 1, 128, *st, *tail) == V.MLA_ERR_ARG
    assert lib.mla_rope_apply(r, FAKE, FAKE, FAKE, 3, 1, 1, 128, *st, *tail) == V.MLA_ERR_ARG
    assert lib.mla_rope_apply(r, FAKE, FAKE, FAKE, 0, -1, 1, 128, *st, *tail) == V.MLA_ERR_ARG
    assert lib.mla_rope_apply(r, FAKE, FAKE, FAKE, 0, 1, 0, 128, *st, *tail) == V.MLA_ERR_ARG
    assert lib.mla_rope_apply(r, FAKE, FAKE, FAKE, 0, 1, 1, 31, *st, *tail) == V.MLA_ERR_ARG
    assert lib.mla_rope_apply(r, ODD, FAKE, FAKE, 2, 1, 1, 128, *st, *tail) == V.MLA_ERR_ARG
    assert lib.mla_rope_apply(r, FAKE, FAKE, FAKE, 0, 1, 1, 128, 128, 128, 256, 128,
                              *tail) == V.MLA_ERR_ARG       # in place, other strides
    assert lib.mla_rope_apply(r, None, None, None, 0, 0, 1, 128, *st, *tail) == V.MLA_OK


@pytest.mark.parametrize("kind,name,factor", [(0, "none", 1.0), (1, "linear", 4.0),
                                              (2, "ntk", 8.0), (3, "yarn", 4.0),
                                              (3, "yarn", 1.0)])
@pytest.mark.parametrize("dim", [4, 64])
def test_scaled_table(kind, name, factor, dim):
    """cos and sin in double, rounded once: half a unit of the last place of
    values up to 1.21 (YaRN's factor at 8) is 2^-24; the angle in double is
    exact to 1e-12 at these positions."""
    tab = V.mla_rope_scaled_table_fill(dim, 4096, 10000.0, kind, factor, native_len=1024)
    f, size = O.scaled_freqs(dim, 10000.0, name, factor, 1024)
    ang = np.arange(4096)[:, None] * f
    np.testing.assert_allclose(tab[..., 0], np.cos(ang) * size, rtol=0, atol=2 ** -23)
    np.testing.assert_allclose(tab[..., 1], np.sin(ang) * size, rtol=0, atol=2 ** -23)


def test_scaled_table_refusals():
    good = dict(rot_dim=64, table_len=16, theta=1e4, scaling=3, factor=4.0, native_len=1024)
    V.mla_rope_scaled_table_fill(**good)
    for bad in (dict(rot_dim=63), dict(rot_dim=0), dict(table_len=0), dict(theta=0.0),
                dict(theta=float("nan")), dict(scaling=4), dict(scaling=-1), dict(factor=0.5),
                dict(factor=float("inf")), dict(native_len=0), dict(beta_fast=1.0),
                dict(scaling=2, rot_dim=2)):
        with pytest.raises(V.MlaError) as e:
            V.mla_rope_scaled_table_fill(**{**good, **bad})
        assert e.value.code == V.MLA_ERR_ARG


def test_oracle_pages_stay_consistent():
    """Random operations: every page's count equals the streams that name it,
    and a stream's rows are what was appended to it, whatever others did."""
    rng = np.random.default_rng(5)
    o = O.Pages(1, 40, 8, 6, 12, 8, 8)
    want = {s: np.zeros((0, 8)) for s in range(6)}
    for step in range(300):
        kind = rng.integers(4)
        if kind == 0:
            s = int(rng.integers(6))
            n = int(rng.integers(1, 20))
            new = np.full(6, -1)
            new[s] = o.lens[s] + n
            before = int(o.lens[s])
            o.resize(new)
            if o.lens[s] == before + n:
                rows = rng.standard_normal((n, 8))
                q = [0] * (s + 1) + [n] * (6 - s)
                o.append(0, rows, rows, q)
                want[s] = np.concatenate([want[s], rows])
        elif kind == 1:
            s = int(rng.integers(6))
            new = np.full(6, -1)
            new[s] = int(rng.integers(0, o.lens[s] + 1))
            o.resize(new)
            want[s] = want[s][:new[s]]
        elif kind == 2:
            a, b = (int(v) for v in rng.permutation(6)[:2])
            if o.lens[b] == 0:
                o.fork([a], [b])
                want[b] = want[a].copy()
        else:
            o.compact()
            used = np.flatnonzero(o.refs)
            assert list(used) == list(range(len(used)))
        count = np.bincount(o.table[o.table >= 0], minlength=40)
        assert np.array_equal(count, o.refs)
        for s in range(6):
            assert np.array_equal(o.rows(0, s)[0], want[s]), (step, s)
