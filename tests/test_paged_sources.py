"""How the kernels of the paged cache and the rotation read their inputs, checked in the
sources (no GPU needed).

They start while the stream's previous kernel still runs, and neighbouring calls write
what the next one reads: lengths, page tables and reference counts, latents, queries.
Loads through the non-coherent path (__ldg, ld.global.nc, const __restrict__ parameters)
may only be used for data that nothing writes while the kernel runs, its early start
included, so none of these files has one."""

import os
import re

import pytest

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))),
                    "paper_2605_30351_gb300", "csrc")


@pytest.mark.parametrize("name", ["paged_common.cuh", "paged_attn.cuh", "paged_attn.cu",
                                  "paged_decode.cu", "paged_append.cu", "pages.cu", "rope.cu"])
def test_inputs_are_read_coherently(name):
    with open(os.path.join(CSRC, name)) as f:
        code = re.sub(r"//[^\n]*", "", f.read())
    assert not re.findall(r"__ldg|\.nc\b|__restrict__|__ldca", code)
