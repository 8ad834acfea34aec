"""Naming a form of attention over a window, no GPU needed."""

import ctypes

import pytest

from paper_2605_30351_gb300 import videomla as V


def test_forms():
    lib = V.load()
    for form in (1, 2, 4, 8, 16, 128, 256, 0):
        assert lib.mla_selftest_window_form(form, None) == V.MLA_OK
    taken = ctypes.c_int(-7)
    assert lib.mla_selftest_window_form(0, ctypes.byref(taken)) == V.MLA_OK and taken.value >= 0


@pytest.mark.parametrize("form", [-1, 3, 5, 6, 7, 9, 15, 17, 32, 64, 127, 129, 512, 1 << 30])
def test_others_are_refused(form):
    taken = ctypes.c_int(-7)
    assert V.load().mla_selftest_window_form(form, ctypes.byref(taken)) == V.MLA_ERR_ARG
    assert taken.value == -7
