// Single tokens and short tiles over their streams' sinks and sliding window: instances of
// paged_decode_kernel.cuh.
#include "paged_decode_kernel.cuh"

namespace vmla {

int launch_window_teams(const PagedAttnArgs& a, int team, int teams) {
  return a.d_r == 32 ? pick_teams<32>(a, team, teams) : pick_teams<64>(a, team, teams);
}

int window_team_slots(int team) { return team_slots<192, 32>(team); }

int launch_window_decode(const PagedAttnArgs& a) {
  return a.d_r == 32 ? pick_decode<32, true>(a) : pick_decode<64, true>(a);
}

}  // namespace vmla
