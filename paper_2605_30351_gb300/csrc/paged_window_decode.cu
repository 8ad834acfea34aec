// Single tokens and short tiles over their streams' sinks and sliding window: instances of
// paged_decode_kernel.cuh.
#include "paged_decode_kernel.cuh"

namespace vmla {

int launch_window_decode(const PagedAttnArgs& a) {
  return a.d_r == 32 ? pick_decode<32, true>(a) : pick_decode<64, true>(a);
}

}  // namespace vmla
