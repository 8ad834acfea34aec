// Attention of ragged streams' newest tokens over the sinks and the sliding window of a
// paged latent cache (Eq. score; App. D.4, D.5, E): the choice of a kernel.
#include <algorithm>
#include <atomic>
#include <numeric>

#include "paged_attn_kernel.cuh"

namespace vmla {
namespace {

// A window bounds what a tile of 16 rows needs, so the host knows how many key blocks of 128
// that may be, and whether a team of a few CTAs is done with it sooner than shares of all
// tiles' blocks and their join, a second launch. Estimates in tenths of a us, from calls with
// 64 sinks and pages of 64 tokens at d_c = 192, used at every width; the clusters that run at a
// time are asked of d_c = 192's instance, which has one CTA an SM (d_c = 64's could have two).
//   teams   a wave of them takes 7 us and 1.4 a block, whatever the others do, 0.5 more where
//           streams may have more than one tile; teams of more than one CTA 1.2 more in all
//   shares  11.5 us, 1.4 for the blocks that each SM has on average and 3 for its tiles
//   tiles of 128 rows (streams of more than 16 rows on average)  16 us and 1.2 a block
// Blocks are what the windows bound; shares, and more so tiles of 128 rows, gain where streams
// are shorter, and the estimates are fitted to such calls too. Of 400 other calls, drawn (1 - 17
// tokens of 1 - 300 streams, whole and ragged, 50 for each d_c and d_r), every form was timed: the
// choice takes longer than the best by 1.3 and 1.7 % on average at d_c = 64 with d_r = 32 and 64,
// 2.6 and 2.2 at 128, 3.2 and 2.6 at 192, 2.4 and 5.2 at 256, at most by 46; always shares 28 %,
// always tiles of 128 rows 27, always teams of one CTA 66. Farthest off: a token or two of some 200
// streams. Every slot of the pool counts as a stream with work, as the host does not know which
// are idle.
// Measured, one token of n streams, window w (teams of 8, 4, 2, 1: the best; shares):
//   n = 1, w = 300: 8.8, 10.6   n = 12, w = 2,000: 12.0, 13.7  n = 76, w = 1,000: 17.7, 23.3
//   n = 1, w = 4,000: 13.7, 11.5  n = 38, w = 4,000: 34.4, 27.4  n = 96, w = 300: 11.4, 14.5
// and tiles of 16 or 128 rows: 5 tokens of 4 streams, 16 heads, w = 300: 10.4, 15.3; of 40:
// 22.5, 17.0.
int team_of(const PagedAttnArgs& a, bool tall, int& teams) {
  const long long rows = static_cast<long long>(a.total) * a.heads;
  const long long most = rows / 16 + a.seqs;  // teams that may find work
  if (a.form != 0) {
    const int slots = a.form <= 8 ? window_team_slots(a.form) : 0;
    teams = static_cast<int>(std::min<long long>(slots, most));
    return slots > 0 ? a.form : 0;
  }
  const long long page = a.page_tokens, bn = 128;
  const bool divides = bn % page == 0;
  // the window of a tile's tokens, ends in pages
  const long long seen = (a.sinks + page - 1) / page * page + a.window + 15 / a.heads + page - 1;
  const long long keys = std::min(seen, static_cast<long long>(a.max_pages) * page);
  const long long blocks =
      divides ? (keys + bn - 1) / bn : (keys / page + 2) * ((page + bn - 1) / bn);
  const long long streams = std::min(a.seqs, a.total);
  const bool further = a.total > a.seqs || a.heads > 16;
  // of 16 rows: exact where streams have as many tokens each, else as far as rows fill the
  // last tile of each on average, and some for streams that idle
  const long long last = streams * (16 - std::gcd(a.heads, 16)) / 32 + streams / 8 + 1;
  const long long all =
      a.total % streams == 0 ? streams * ((rows / streams + 15) / 16) : rows / 16 + last;
  const long long tiles = std::max<long long>(a.seqs, further ? all : 0);
  long long best = tall ? 160 + 12 * a.seqs * blocks / kMaxCtas
                        : 115 + (30 + 14 * blocks) * a.seqs / kMaxCtas;
  int team = 0;
  for (int t = 8; t > 0; t /= 2) {
    const int slots = window_team_slots(t);
    if (slots < 1) continue;
    const long long waves = (tiles + slots - 1) / slots;
    const long long cost =
        waves * (70 + (further ? 5 : 0) + 14 * ((blocks + t - 1) / t)) + (t > 1 ? 12 : 0);
    if (cost < best) {
      best = cost;
      team = t;
      teams = static_cast<int>(std::min<long long>(slots, most));
    }
  }
  return team;
}

// mla_selftest_window_form: what is asked for, and what the last call took
std::atomic<int> asked_form{0}, taken_form{0};

}  // namespace

int window_form(int form, int* taken) {
  switch (form) {
    case 0:
    case 1:
    case 2:
    case 4:
    case 8:
    case 16:
    case kBM:
    case 2 * kBM: break;
    default: return MLA_ERR_ARG;
  }
  asked_form = form;
  if (taken) *taken = taken_form;
  return MLA_OK;
}

int launch_paged_window_attention(const PagedAttnArgs& call) {
  PagedAttnArgs a = call;
  a.form = asked_form;
  const bool short_forms = a.d_c <= 256;  // d_c = 512 has tiles of 128 rows only
  if (a.form != 0 && !short_forms && a.form != kBM) return MLA_ERR_UNSUPPORTED;
  const bool tall = a.form != 0 ? a.form >= kBM
                                : static_cast<long long>(a.total) * a.heads > 16ll * a.seqs;
  if (short_forms) {
    int teams = 0;
    const int team = team_of(a, tall, teams);
    if (team > 0) {
      taken_form = team;
      return launch_window_teams(a, team, teams);
    }
    if (a.form != 0 && a.form <= 8) return MLA_ERR_UNSUPPORTED;
    if (!tall) {
      taken_form = 16;
      return launch_window_decode(a);
    }
  }
  taken_form = short_forms && takes_pairs(a) ? 2 * kBM : kBM;
  return a.d_r == 32 ? pick_dc<32, true>(a) : pick_dc<64, true>(a);
}

}  // namespace vmla
