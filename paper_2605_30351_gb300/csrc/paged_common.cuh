// Device helpers of the paged-cache kernels.
//
// These kernels start while the previous one of the stream still runs, and that one may
// write any of their inputs (lengths, tables, latents, queries): they read them with
// plain loads after grid_dep_sync, never through the non-coherent path, which asks for
// data that nothing writes while the kernel is there.
#pragma once

#include <cuda_runtime.h>

#include "ptx_sm103.cuh"

namespace vmla {

// The last stream whose first token is not past t: every lane gets the answer.
__device__ __forceinline__ int stream_of(const int* q_start, int seqs, int t, int lane) {
  int lo = 0, n = seqs;
  while (n > 1) {
    const int step = (n + 31) / 32;
    const int at = lane * step;
    const bool le = at < n && q_start[lo + at] <= t;
    const unsigned m = __ballot_sync(0xffffffffu, le);
    const int k = m ? 31 - __clz(m) : 0;
    lo += k * step;
    n = min(step, n - k * step);
  }
  return lo;
}

// Record a q_start that does not ascend from 0 to total; one block calls it.
__device__ __forceinline__ void check_q_start(const int* q_start, int seqs, int total,
                                              int* status) {
  for (int s = threadIdx.x; s <= seqs; s += blockDim.x) {
    const int v = q_start[s];
    const int next = s < seqs ? q_start[s + 1] : total;
    if (v > next || (s == 0 && v != 0) || (s == seqs && v != total))
      record_status(status, MLA_ERR_RANGE);
  }
}

}  // namespace vmla
