"""How many teams of a size run at a time is asked of the CUDA runtime. A question that fails
leaves that size out, and the call goes on and succeeds: it must not leave its error behind as
that of the last MLA_ERR_CUDA return. The runtime's answers are made up here (no GPU needed)."""

import os
import subprocess

import pytest

from paper_2605_30351_gb300 import build as B

SOURCE = r"""
#include <cstdio>
#include <cuda_runtime.h>

static cudaError_t answer = cudaSuccess;
static int asked = 0, recorded = 0;
static cudaError_t fake_device(int* d) { *d = 0; return cudaSuccess; }
template <typename F> cudaError_t fake_attribute(F, cudaFuncAttribute, int) { return cudaSuccess; }
template <typename F> cudaError_t fake_clusters(int* n, F, cudaLaunchConfig_t*) {
  ++asked;
  if (answer == cudaSuccess) *n = 1000;
  return answer;
}
#define cudaGetDevice fake_device
#define cudaFuncSetAttribute fake_attribute
#define cudaOccupancyMaxActiveClusters fake_clusters
#include "paged_decode_kernel.cuh"

namespace vmla {
void set_last_cuda_error(cudaError_t) { ++recorded; }
int slots(int team) { return team_slots<192, 32>(team); }
}

int main() {
  answer = cudaErrorInvalidValue;
  const int a = vmla::slots(8), b = vmla::slots(2);
  answer = cudaSuccess;
  const int c = vmla::slots(8), d = vmla::slots(1);
  answer = cudaErrorInvalidValue;
  const int e = vmla::slots(8), f = vmla::slots(2);
  std::printf("%d %d %d %d %d %d asked %d recorded %d\n", a, b, c, d, e, f, asked, recorded);
}
"""


def test_a_failed_question_leaves_no_error(tmp_path):
    try:
        nvcc = B._nvcc()
    except RuntimeError:
        pytest.skip("no nvcc")
    src, exe = tmp_path / "slots.cu", tmp_path / "slots"
    src.write_text(SOURCE)
    r = subprocess.run([nvcc, *B.ARCH, *B.NVCC_FLAGS, "-o", str(exe), str(src)], capture_output=True, text=True)
    assert r.returncode == 0, r.stderr
    r = subprocess.run([str(exe)], capture_output=True, text=True, timeout=60)
    # of 152 CTAs: 19 teams of eight; a size once known is not asked for again, one that failed is
    assert r.stdout == "0 0 19 152 19 0 asked 5 recorded 0\n", r.stdout + r.stderr
