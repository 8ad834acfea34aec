// Attention of ragged streams' newest tokens over the sinks and the sliding window of a
// paged latent cache (Eq. score; App. D.4, D.5, E): the choice of a kernel.
#include "paged_attn_kernel.cuh"

namespace vmla {

int launch_paged_window_attention(const PagedAttnArgs& a) {
  if (a.d_c <= 256 && static_cast<long long>(a.total) * a.heads <= 16ll * a.seqs)
    return launch_window_decode(a);
  return a.d_r == 32 ? pick_dc<32, true>(a) : pick_dc<64, true>(a);
}

}  // namespace vmla
