// Single tokens and short tiles over all tokens that their streams hold: instances of
// paged_decode_kernel.cuh.
#include "paged_decode_kernel.cuh"

namespace vmla {

int launch_paged_decode(const PagedAttnArgs& a) {
  return a.d_r == 32 ? pick_decode<32, false>(a) : pick_decode<64, false>(a);
}

}  // namespace vmla
