"""Host side of attention over the paged latent cache, no GPU needed: the size of
its workspace and its argument rules, all of them checked before any pointer is
used."""

import ctypes

import pytest

from paper_2605_30351_gb300 import videomla as V

FAKE = 1 << 20


def paged(**kw):
    a = dict(c=FAKE, kr=FAKE, table=FAKE, lens=FAKE, refs=FAKE, plan=FAKE, layers=2, pages=64,
             page_tokens=16, seqs=3, max_pages=8, d_c=192, d_r=32)
    a.update(kw)
    return V.mla_paged_cache(**a)


def call(cache=None, **kw):
    a = dict(layer=0, q_c=FAKE, q_r=FAKE, total=4, heads=12, q_start=FAKE, head_dim=128, block=1,
             workspace=FAKE, nbytes=1 << 30, o=FAKE, stream=None)
    a.update(kw)
    c = paged() if cache is None else cache
    return V.load().mla_paged_attention(ctypes.byref(c), *a.values())


@pytest.mark.parametrize("d_r", [32, 64])
@pytest.mark.parametrize("d_c,d_v", [(64, 64), (128, 128), (192, 192), (256, 256), (512, 256)])
def test_workspace_has_room_to_start_on_a_32_byte_boundary(d_c, d_v, d_r):
    """Two slots for each of 152 CTAs: 128 partial rows of d_v fp32 values, stored 32
    bytes at a time, with their maximum and sum, and a 16-byte descriptor. The
    caller's workspace may start at any 16-byte boundary, so 16 more."""
    c = paged(d_c=d_c, d_r=d_r)
    layout = 2 * 152 * (128 * (4 * d_v + 8) + 16)
    assert V.load().mla_paged_workspace_bytes(ctypes.byref(c)) >= layout + 16


@pytest.mark.parametrize("bad", [
    dict(layer=2), dict(layer=-1), dict(total=-1), dict(heads=0), dict(heads=-1),
    dict(head_dim=0), dict(block=-1), dict(total=1 << 20, heads=(1 << 10) + 1),
    dict(q_c=None), dict(q_r=None), dict(q_start=None), dict(workspace=None), dict(o=None),
    dict(q_c=FAKE + 8), dict(q_r=FAKE + 8), dict(q_start=FAKE + 2), dict(workspace=FAKE + 8),
    dict(o=FAKE + 8), dict(nbytes=0)])
def test_arguments_are_checked(bad):
    assert call(**bad) == V.MLA_ERR_ARG


def test_a_workspace_one_byte_short_is_refused():
    need = V.load().mla_paged_workspace_bytes(ctypes.byref(paged()))
    assert call(nbytes=need - 1) == V.MLA_ERR_ARG


@pytest.mark.parametrize("bad", [dict(c=None), dict(kr=FAKE + 8), dict(table=None),
                                 dict(lens=FAKE + 4), dict(refs=None), dict(seqs=0),
                                 dict(page_tokens=7)])
def test_the_cache_is_checked(bad):
    assert call(paged(**bad)) == V.MLA_ERR_ARG
    assert call(paged(**bad), total=0) == V.MLA_ERR_ARG


@pytest.mark.parametrize("d_c,d_r", [(96, 32), (384, 32), (192, 16), (192, 128)])
def test_widths_without_a_kernel(d_c, d_r):
    c = paged(d_c=d_c, d_r=d_r)
    assert V.load().mla_paged_workspace_bytes(ctypes.byref(c)) == 0
    assert call(c) == V.MLA_ERR_UNSUPPORTED
