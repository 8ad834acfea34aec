// Attention of ragged streams' newest tokens over the sinks and the sliding window of a
// paged latent cache (Eq. score; App. D.4, D.5, E): the choice of a kernel.
#include <algorithm>

#include "paged_attn_kernel.cuh"

namespace vmla {
namespace {

// A window bounds what a tile of 16 rows needs, so the host knows how many key blocks of 128
// that may be, and whether a team of a few CTAs is done with it sooner than shares of all
// tiles' blocks and their join, a second launch. Estimates in tenths of a us, from calls with
// 64 sinks and pages of 64 tokens at d_c = 192; at d_c = 64 and 256 all of them move together.
//   teams   a wave of them takes 7 us and 1.5 a block, whatever the others do; 1.3 more where
//           streams may have more than one tile
//   shares  11 us and 1.8 for the blocks that each SM has on average
//   tiles of 128 rows (streams of more than 16 rows on average)  15 us and 4 a block
// The last two count four fifths of what the windows bound: they gain where streams are
// shorter, while a wave of teams waits for its longest.
// Measured, one token of n streams, window w (teams of 8, 4, 2, 1: the best; shares):
//   n = 1, w = 300: 8.4, 10.5   n = 12, w = 2,000: 11.4, 13.9   n = 76, w = 1,000: 17.0, 19.9
//   n = 1, w = 4,000: 13.3, 11.4   n = 38, w = 4,000: 33.6, 26.0  n = 96, w = 300: 10.8, 17.3
// and tiles of 16 or 128 rows: 5 tokens of 4 streams, 16 heads, w = 300: 10.4, 15.3; of 40:
// 22.5, 17.0.
int team_of(const PagedAttnArgs& a, bool tall, int& teams) {
  const long long rows = static_cast<long long>(a.total) * a.heads;
  const long long page = a.page_tokens, bn = 128;
  const bool divides = bn % page == 0;
  // the window of a tile's tokens, ends in pages
  const long long seen = (a.sinks + page - 1) / page * page + a.window + 15 / a.heads + page - 1;
  const long long keys = std::min(seen, static_cast<long long>(a.max_pages) * page);
  const long long blocks =
      divides ? (keys + bn - 1) / bn : (keys / page + 2) * ((page + bn - 1) / bn);
  const long long streams = std::min(a.seqs, a.total);
  const bool further = a.total > a.seqs || a.heads > 16;
  const long long tiles = std::max<long long>(a.seqs, further ? rows / 16 + streams / 2 : 0);
  long long best = tall ? 150 + 32 * a.seqs * blocks / kMaxCtas
                        : 110 + 14 * a.seqs * blocks / kMaxCtas;
  int team = 0;
  for (int t = 8; t > 0; t /= 2) {
    const int slots = window_team_slots(t);
    if (slots < 1) continue;
    const long long waves = (tiles + slots - 1) / slots;
    const long long cost = waves * (70 + (further ? 13 : 0) + 15 * ((blocks + t - 1) / t));
    if (cost < best) {
      best = cost;
      team = t;
      teams = static_cast<int>(std::min<long long>(slots, rows / 16 + a.seqs));
    }
  }
  return team;
}

}  // namespace

int launch_paged_window_attention(const PagedAttnArgs& a) {
  const bool tall = static_cast<long long>(a.total) * a.heads > 16ll * a.seqs;
  if (a.d_c <= 256) {
    int teams = 0;
    const int team = team_of(a, tall, teams);
    if (team > 0) return launch_window_teams(a, team, teams);
    if (!tall) return launch_window_decode(a);
  }
  return a.d_r == 32 ? pick_dc<32, true>(a) : pick_dc<64, true>(a);
}

}  // namespace vmla
