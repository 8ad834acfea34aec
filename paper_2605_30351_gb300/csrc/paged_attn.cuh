// What the kernels of attention over a paged cache share: parameters, the split of
// the work into shares, and the places of partial results.
#pragma once

#include "internal.h"
#include "paged_common.cuh"

namespace vmla {

constexpr int kBM = 128;       // rows of a partial tile's slot
constexpr int kMaxCtas = 152;  // the workspace holds two slots for each

// Workspace of a call whose CTAs hold dv output columns: partial rows (fp32), their
// (maximum, sum), and a descriptor per slot. Partial rows are stored 32 bytes at a
// time, while the caller's workspace starts on any 16-byte boundary: the layout
// starts at the next 32-byte one, so a workspace has 16 bytes to spare.
struct PartLayout {
  unsigned long long ml, desc, total;
  explicit PartLayout(int dv)
      : ml(2ull * kMaxCtas * kBM * dv * 4),
        desc(ml + 2ull * kMaxCtas * kBM * 8),
        total(desc + 2ull * kMaxCtas * 16 + 16) {}
  static char* base(void* workspace) {
    return reinterpret_cast<char*>((reinterpret_cast<unsigned long long>(workspace) + 31) & ~31ull);
  }
};

// Places of the pages that hold a stream's sinks; past the largest index they are all alike.
inline int sink_places(int sinks, int page_tokens) {
  const long long n = (static_cast<long long>(sinks) + page_tokens - 1) / page_tokens * page_tokens;
  return static_cast<int>(n < kMostTokens ? n : kMostTokens);
}

// What a short call pays for is the code that it runs for the first time, about 15
// ns an instruction: divisions by the call's own numbers are prepared on the host.
// n / d for 0 <= n < 2^31 and d >= 1: mul = floor(2^shift / d) + 1 with shift = 31 +
// ceil(log2 d), so the error of n * mul / 2^shift, at most n / 2^shift, stays below
// the next multiple of 1 / d.
struct Div {
  unsigned mul;
  int shift;
  __device__ __forceinline__ int operator()(int n) const {
    return static_cast<int>((static_cast<unsigned long long>(n) * mul) >> shift);
  }
};
inline Div div_by(int d) {
  int s = 0;
  while ((1ll << s) < d) ++s;
  return Div{static_cast<unsigned>((1ull << (31 + s)) / static_cast<unsigned>(d) + 1), 31 + s};
}

struct PagedK {
  const int* q_start;
  const int* table;
  const int* lens;
  __nv_bfloat16* o;
  float* part_o;
  float2* part_ml;
  int4* part_desc;  // first row in o, rows, kPart*, 1 or 2 = row after row
  int total, heads, seqs, pages, page_tokens, max_pages, block;
  // Key blocks never straddle a group of `group` tokens: BN tokens (per_group
  // whole pages) where the pages divide a block, else one page.
  int group, blocks, per_group;
  int box_rows;
  Div by_heads, by_group, by_blocks, by_mask;  // by_mask: by `block`
  float scale_log2;
  int* status;
};

// The same with a window that slides (WIN, here and below).
template <bool WIN>
struct PagedP : PagedK {};
template <>
struct PagedP<true> : PagedK {
  // tokens given back by stream (or none), the window, the sinks and the places of their whole
  // pages; q_r of its own for the sinks
  const int* dropped;
  int window, sinks, front;
  bool turned;
  // pages divide a key block (they are a power of two of tokens): blocks are runs of pages
  // wherever these lie
  bool compact;
  int page_log;  // log2 of page_tokens where they do, else 0
  bool o_wide;   // o's rows start on 32-byte boundaries
};

// Partial rows lie as [4 columns][128 rows], which a warp (a lane per row) writes in
// full lines, except those of short tiles (up to 32 rows) and of tiles that more than
// four shares cut: they lie row after row, as the join reads them, a warp or
// (part_desc.w = 2: tiles of more than four shares, and all of paged_decode.cu) a
// block for each row. Two or eight shares instead of four: 100 new tokens of 9 ragged
// streams 28.9 or 25.9 us (25.9), 5 drafted tokens of 16 streams at d_c = 512 43.6 or
// 46.8 us (44.4).
constexpr int kFewRows = 32;
constexpr int kManyShares = 4;

// part_desc.z: the slot holds a partial tile, that ends its tile; the CTA's share
// is empty (a chain of partial tiles passes over it)
constexpr int kPartHeld = 1, kPartEnds = 2, kPartEmpty = 4;

// The maximum of a partial row is -inf only where the row sees none of the part's keys,
// and the join passes over those (their values are whatever 0 times a hidden key's is).
// Where every key seen scores -inf or NaN it is the lowest finite number, so that a NaN
// sum or value gets into the row whatever its weight.
constexpr float kLowest = -3.402823466e38f;

template <bool WIN>
struct Stream {
  int q0, n, len;
  static constexpr int gone = 0;
};
template <>
struct Stream<true> {
  int q0, n, len, gone;
};

template <bool WIN>
__device__ __forceinline__ bool stream_held(const PagedP<WIN>& p, int n, int len, int gone) {
  if (len < 0 || len > static_cast<long long>(p.max_pages) * p.page_tokens) return false;
  if constexpr (WIN)  // indices below the limit, and new tokens behind the sinks' pages
    return gone >= 0 && static_cast<long long>(len) + gone < kMostTokens &&
           (gone == 0 || static_cast<long long>(len) - n >= p.front);
  return true;
}

template <bool WIN>
__device__ __forceinline__ Stream<WIN> stream_at(const PagedP<WIN>& p, int s) {
  Stream<WIN> t{p.q_start[s], p.q_start[s + 1], p.lens[s]};
  const int q1 = t.n;
  t.n = q1 - t.q0;
  // The two tests say the same without a window; but through stream_held the compiler orders
  // the block loop at d_c = 512, d_r = 64 so that it takes 3 - 6 % longer (429 tokens of 3
  // streams on 18,367 keys: 496 us, 466 so).
  if constexpr (WIN) {
    t.gone = p.dropped ? p.dropped[s] : 0;
    if (t.q0 < 0 || q1 < t.q0 || q1 > p.total || !stream_held<WIN>(p, t.n, t.len, t.gone)) t.n = 0;
  } else {
    if (t.q0 < 0 || q1 < t.q0 || q1 > p.total || t.len < 0 ||
        t.len > static_cast<long long>(p.max_pages) * p.page_tokens)
      t.n = 0;
  }
  return t;
}

// Record lengths that the table cannot hold (and what else stream_held asks for, of
// streams with new tokens), and a q_start that does not ascend; `threads` threads of one block
// call it, of which this is the i-th.
template <bool WIN>
__device__ __forceinline__ void check_streams(const PagedP<WIN>& p, int i, int threads) {
  check_q_start(p.q_start, p.seqs, p.total, p.status, i, threads);
  for (int s = i; s < p.seqs; s += threads) {
    int n = 0, gone = 0;
    if constexpr (WIN) {
      n = p.q_start[s + 1] - p.q_start[s];
      if (p.dropped && n > 0) gone = p.dropped[s];
    }
    if (!stream_held<WIN>(p, n, p.lens[s], gone)) record_status(p.status, MLA_ERR_RANGE);
  }
}

// Where the keys end that the token at place a (it may be negative) of a stream sees:
// blocks of the mask count from the stream's start.
template <bool WIN>
__device__ __forceinline__ int keys_seen(const PagedP<WIN>& p, int a, const Stream<WIN>& st) {
  if (a < 0) return 0;
  if (p.block == 0) return st.len;
  const long long end = static_cast<long long>(p.by_mask(a + st.gone) + 1) * p.block - st.gone;
  return end < st.len ? static_cast<int>(end) : st.len;
}

// The first key behind the sinks that a token sees whose keys end there.
__device__ __forceinline__ int first_key(const PagedP<true>& p, int keys, int gone) {
  return max(gone > 0 ? p.front : p.sinks, keys - p.window);
}

// Key blocks before place `keys`, the one it lies in included.
template <int BN>
__device__ __forceinline__ int blocks_to(const PagedK& p, int keys) {
  const int whole = p.by_group(keys), rest = keys - whole * p.group;
  return whole * p.blocks + (rest + BN - 1) / BN;
}

// The key blocks of row tile `tile` (TR rows) of a stream: what its last row, which sees
// most, needs; at least one, so that rows that see nothing are written.
//
// With a window, what a tile needs is its sinks' pages and the pages from the first key of
// its first row on. Where pages divide a block they follow one another without a gap: the
// tile counts its tokens through, u < cut are the sinks' pages, from cut on the token u lies
// at place u + shift (blocks of 9 ragged prompts, 16 tokens a page and a window of 1,024:
// 9 a tile instead of 10). Sinks with queries of their own end at a multiple of 16 tokens, as
// the columns of an MMA do, else of a block. Where pages do not divide a block (cut = shift =
// 0) the blocks are two runs of the stream's: 0 .. sb - 1 with the sinks, then from wb on;
// a block that holds sinks and window keys is in both runs where the sinks have queries of
// their own, else in the first. sb: blocks that hold sinks, in both cases.
template <bool WIN>
struct Span {
  int all;
  static constexpr int sb = 0, wb = 0, cut = 0, shift = 0;
};
template <>
struct Span<true> {
  int all, sb, wb, cut, shift;
};

template <int BN, int TR, bool WIN>
__device__ __forceinline__ Span<WIN> tile_span(const PagedP<WIN>& p, const Stream<WIN>& st, int tile) {
  const int last = min(st.n * p.heads, (tile + 1) * TR) - 1;
  const int keys = keys_seen<WIN>(p, st.len - st.n + p.by_heads(last), st);
  if constexpr (!WIN) {
    return Span<WIN>{max(1, blocks_to<BN>(p, keys))};
  } else {
    const int low =
        first_key(p, keys_seen<WIN>(p, st.len - st.n + p.by_heads(tile * TR), st), st.gone);
    const int sink_end = min(p.sinks, keys);
    Span<WIN> v{0, 0, 0, 0, 0};
    if (p.compact) {
      const int sp = (sink_end + p.page_tokens - 1) >> p.page_log;
      if (keys > low) {
        int wp = low >> p.page_log;
        if (!p.turned) wp = max(wp, sp);
        v.cut = sp << p.page_log;
        if (p.turned && v.cut % 16) v.cut = (v.cut + BN - 1) / BN * BN;
        v.shift = (wp << p.page_log) - v.cut;
        v.all = max(1, (keys - v.shift + BN - 1) / BN);
        v.sb = (v.cut + BN - 1) / BN;
      } else {  // sinks only
        v.sb = (sink_end + BN - 1) / BN;
        v.cut = v.sb * BN;
        v.all = max(1, v.sb);
      }
      v.wb = v.sb;
    } else {
      v.sb = blocks_to<BN>(p, sink_end);
      int n = 0;
      if (keys > low) {
        const int grp = p.by_group(low);
        v.wb = grp * p.blocks + (low - grp * p.group) / BN;
        if (!p.turned) v.wb = max(v.wb, v.sb);
        n = max(0, blocks_to<BN>(p, keys) - v.wb);
      }
      v.all = max(1, v.sb + n);
    }
    return v;
  }
}

// Cost of a stream's row tiles in keys, as a straight line from the first to the
// last tile's keys (exact for a whole chunk and token by token, and within a
// mask block for others) plus kTileCost for loading Q and writing O: prefix sums
// in closed form, so a share's ends are found without walking the tiles. Four blocks:
// with two or eight the ragged and the drafted tokens' calls are 2 - 8 % slower.
template <int BN>
constexpr int kTileCost = 4 * BN;

// With a window these keys come first, in the share that begins the tile: one that begins
// inside a tile pays for its Q and O too, as nearly all do, and one that begins another tile
// besides pays twice. At the tile's end, spread over its keys, the slowest CTA of 5 drafted
// tokens of 16 streams at d_c = 512 had two tiles and took 29 us, those with one 20.5; the
// call takes 36.9 us so and 33.1 in front, 64 streams of one token 60.8 and 57.8, 66 calls
// of prompts and long windows 5 % less on average. Two or three blocks for tiles of 128 rows
// and two or four for those of 16 differ from these by 1 % on average.
// In shares of few blocks a tile's head in front would leave CTAs without work, and whole blocks
// to the others: only what a share is longer than a block comes in front (of tiles of 128 rows
// twice that), the rest is spread over the keys. One token of one stream on 4,000 keys (d_c = 192)
// 11.3 us so, 12.3 with all of it in front; 20 calls at d_c = 512 2 % less on average.
template <int BN, int TR, bool WIN>
constexpr int kTileHead = !WIN ? kTileCost<BN> : TR > 16 ? 4 * BN : 3 * BN;

template <bool WIN>
struct Cost {
  long long first, slope;  // slope in 1/256 keys per tile
  int tiles;
  __device__ long long before(int t) const {  // of tiles 0 .. t-1
    return t * first + ((slope * (static_cast<long long>(t) * (t - 1) / 2)) >> 8);
  }
};

// With a window the line ends where sinks and window are full, at tile `knee`; from
// there on all tiles cost the same.
template <>
struct Cost<true> {
  long long first, slope, flat;
  int tiles, knee;
  __device__ long long before(int t) const {
    const int k = min(t, knee);
    return k * first + ((slope * (static_cast<long long>(k) * (k - 1) / 2)) >> 8) +
           (t - k) * flat;
  }
};

template <int BN, int TR, bool WIN>
__device__ __forceinline__ Cost<WIN> cost_of(const PagedP<WIN>& p, const Stream<WIN>& st) {
  Cost<WIN> c{};
  if (st.n == 0) return c;
  const int rows = st.n * p.heads;
  c.tiles = (rows + TR - 1) / TR;
  const int k1 = keys_seen<WIN>(p, st.len - 1, st);
  if constexpr (WIN) {
    // what a row sees of k keys is min(k - off, cap): the keys of the sinks' pages that a
    // stream which gave pages back does not see are off
    const int off = st.gone > 0 ? p.front - p.sinks : 0;
    const long long cap = static_cast<long long>(p.sinks) + p.window;
    const int v1 = k1 - off;
    const int v0 = c.tiles > 1
                       ? keys_seen<WIN>(p, st.len - st.n + p.by_heads(TR - 1), st) - off
                       : v1;
    c.flat = min(cap, static_cast<long long>(v1)) + kTileHead<BN, TR, WIN>;
    if (v0 >= c.flat - kTileHead<BN, TR, WIN>) return c;  // all tiles alike: the knee is at 0
    // products below 2^63: slope < 2^39 / tiles, of at most 2^23 tiles
    c.first = v0 + kTileHead<BN, TR, WIN>;
    c.slope = static_cast<long long>(__fdividef((v1 - v0) * 256.f, c.tiles - 1.f));
    c.knee = c.tiles;
    if (v1 > cap)
      c.knee = min(c.tiles, 1 + static_cast<int>(__fdividef((cap - v0) * (c.tiles - 1.f),
                                                           static_cast<float>(v1 - v0))));
  } else {
    c.first = k1 + kTileCost<BN>;
    if (c.tiles > 1) {
      const int k0 = keys_seen<WIN>(p, st.len - st.n + p.by_heads(TR - 1), st);
      if (c.tiles <= 4096) {  // the products stay below 2^63
        c.first = k0 + kTileCost<BN>;
        c.slope = static_cast<long long>(__fdividef((k1 - k0) * 256.f, c.tiles - 1.f));
      } else {
        c.first = (static_cast<long long>(k0) + k1) / 2 + kTileCost<BN>;
      }
    }
  }
  return c;
}

template <bool WIN>
struct Place {
  int s, tile, off;  // stream, row tile, key block
  Span<WIN> at;      // the tile's key blocks
  Stream<WIN> st;
};

// The shares' ends: place of share id's first block and of the one after its
// last. Every thread of the block calls it; scratch: 8 long longs and out: two
// Places in shared memory. Three warps look for each end, all streams among their
// 96 threads: one search's latency, not two, is part of every call. With more slots
// than that, idle ones included, a thread walks several of them in turn: one token of
// 16 streams on 2,000 keys takes 13.9 us with 16 slots, 21 with 96, 115 with 1,024 and
// 908 with 8,192. Returns the cost of a share.
template <int BN, int TR, bool WIN>
__device__ __forceinline__ long long find_share(const PagedP<WIN>& p, int id, int groups,
                                                long long* scratch, Place<WIN>* out) {
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const int e = warp / 3;  // which end; the other warps only wait
  const int per = (p.seqs + 95) / 96;
  const int s0 = (threadIdx.x - e * 96) * per;
  long long mine = 0;
  Stream<WIN> st{};
  Cost<WIN> c{};
  if (e < 2)
    for (int k = 0; k < per; ++k)
      if (s0 + k < p.seqs) {
        st = stream_at<WIN>(p, s0 + k);
        c = cost_of<BN, TR, WIN>(p, st);
        mine += c.before(c.tiles);
      }
  long long x = mine;
#pragma unroll
  for (int d = 1; d < 32; d <<= 1) {
    const long long y = __shfl_up_sync(0xffffffffu, x, d);
    if (lane >= d) x += y;
  }
  if (lane == 31 && e < 2) scratch[warp] = x;
  if (threadIdx.x < 2) out[threadIdx.x].s = p.seqs;  // the end of the work
  __syncthreads();
  const long long total = scratch[0] + scratch[1] + scratch[2];
  const int active = static_cast<int>(min(static_cast<long long>(groups), (total + BN - 1) / BN));
  if (id < active && e < 2) {
    long long base = x - mine;
    for (int w = 3 * e; w < warp; ++w) base += scratch[w];
    // total * (id + e) / active: in 32 bits where it fits (a 64-bit division is a
    // noticeable part of a short call), else without the product's overflow
    long long u;
    if (total < (1 << 24)) {
      u = static_cast<unsigned>(total) * (id + e) / static_cast<unsigned>(active);
    } else {
      const long long q = total / active, r = total - q * active;
      u = q * (id + e) + r * (id + e) / active;
    }
    if (u >= base && u < base + mine) {
      long long rem = u - base;
      int s = s0;
      if (per > 1)
        for (; s < p.seqs; ++s) {
          st = stream_at<WIN>(p, s);
          c = cost_of<BN, TR, WIN>(p, st);
          const long long all = c.before(c.tiles);
          if (rem < all) break;
          rem -= all;
        }
      if (s < p.seqs) {
        int lo = 0, hi = c.tiles - 1;  // the last tile that begins at or before rem
        while (lo < hi) {
          const int mid = (lo + hi + 1) / 2;
          if (c.before(mid) <= rem)
            lo = mid;
          else
            hi = mid - 1;
        }
        const long long at = c.before(lo);
        const Span<WIN> span = tile_span<BN, TR, WIN>(p, st, lo);
        long long in = rem - at, all = c.before(lo + 1) - at;
        if constexpr (WIN) {
          long long head = kTileHead<BN, TR, WIN>;
          head = min(head, (TR > 16 ? 2 : 1) * max(total / active - BN, 0ll));
          in = max(in - head, 0ll);
          all = max(all - head, 1ll);
        }
        const int off = static_cast<int>(
            static_cast<float>(in) *
            __fdividef(static_cast<float>(span.all), static_cast<float>(all)));
        out[e] = Place<WIN>{s, lo, min(off, span.all - 1), span, st};
      }
    }
  }
  __syncthreads();
  return active > 0 ? static_cast<long long>(__fdividef(static_cast<float>(total), active)) : 0;
}

// Walks a share segment by segment: a segment is a run of key blocks of one row
// tile. Every role of the CTA walks it for itself.
template <bool WIN>
struct Segment {
  Stream<WIN> st;
  int s, tile;
  int kb0, kb1;  // key blocks [kb0, kb1) of the tile's
  Span<WIN> at;
};

template <int BN, int TR, bool WIN>
struct Walk {
  const PagedP<WIN>& p;
  Stream<WIN> st;
  int s, tile, off;
  Span<WIN> span;  // all < 0: not known yet
  int end_s, end_tile, end_off;
  __device__ Walk(const PagedP<WIN>& k, const Place<WIN>* ends) : p(k) {
    st = ends[0].st;  // the first segment needs no arithmetic: the search had it all
    s = ends[0].s;
    tile = ends[0].tile;
    off = ends[0].off;
    span = ends[0].at;
    end_s = ends[1].s;
    end_tile = ends[1].tile;
    end_off = ends[1].off;
  }
  __device__ bool next(Segment<WIN>& g) {
    if (s >= p.seqs) return false;
    if (span.all < 0) {
      while (tile * TR >= st.n * p.heads) {  // a stream with new tokens
        if (++s >= p.seqs) return false;
        st = stream_at<WIN>(p, s);
        tile = 0;
      }
      span = tile_span<BN, TR, WIN>(p, st, tile);
    }
    const bool last = s == end_s && tile == end_tile;
    if (s > end_s || (s == end_s && tile > end_tile) || (last && off >= end_off)) return false;
    g.st = st;
    g.s = s;
    g.tile = tile;
    g.kb0 = off;
    g.kb1 = last ? end_off : span.all;
    g.at = span;
    off = 0;
    span.all = -1;
    ++tile;
    return true;
  }
};

// Whole tiles instead of a share, for team `id` of `teams`: the first tile of streams id, id +
// teams, ... and the further tiles of all streams, dealt out in turn from the team after the
// last stream's on, so that a stream of many rows does not wait for one team. Every warp of the
// team's CTAs walks them for itself; most calls have no such tiles, and `more` says so.
template <int BN, int TR>
struct TeamWalk {
  const PagedP<true>& p;
  int id, teams, s;
  int base, before;  // streams from base on, and the further tiles of those before
  long long next_more;
  bool more;
  Stream<true> first;  // stream id, loaded while `more` is found out
  __device__ TeamWalk(const PagedP<true>& k, int i, int n, const Stream<true>& st, bool further)
      : p(k), id(i), teams(n), s(i), base(0), before(0), more(further), first(st) {
    next_more = (i + n - k.seqs % n) % n;
  }
  __device__ int further_of(int stream) const {
    if (stream >= p.seqs) return 0;
    const Stream<true> st = stream_at<true>(p, stream);
    return st.n > 0 ? (st.n * p.heads + TR - 1) / TR - 1 : 0;
  }
  __device__ bool take(Segment<true>& g, const Stream<true>& st, int stream, int tile) {
    g.st = st;
    g.s = stream;
    g.tile = tile;
    g.at = tile_span<BN, TR, true>(p, st, tile);
    return true;
  }
  __device__ bool next(Segment<true>& g) {
    while (s < p.seqs) {
      const Stream<true> st = s == id ? first : stream_at<true>(p, s);
      s += teams;
      if (st.n > 0) return take(g, st, s - teams, 0);
    }
    const int lane = threadIdx.x & 31;
    while (more && base < p.seqs) {
      const int mine = further_of(base + lane);
      int x = mine;
#pragma unroll
      for (int d = 1; d < 32; d <<= 1) {
        const int y = __shfl_up_sync(0xffffffffu, x, d);
        if (lane >= d) x += y;
      }
      const int all = __shfl_sync(0xffffffffu, x, 31);
      const long long at = next_more - before;  // among these 32 streams' tiles
      if (at < all) {
        const int l = __ffs(__ballot_sync(0xffffffffu, at < x)) - 1;
        const int first = __shfl_sync(0xffffffffu, x - mine, l);
        next_more += teams;
        return take(g, stream_at<true>(p, base + l), base + l,
                    1 + static_cast<int>(at) - first);
      }
      before += all;
      base += 32;
    }
    return false;
  }
};

// Place of key block kb of the pool's: its first token, and the rows of its group from
// there. The blocks of a segment follow one another from first_block on.
template <int BN>
struct BlockPos {
  int grp, sub;
  __device__ BlockPos(const PagedK& p, int kb) : grp(p.by_blocks(kb)), sub(kb - grp * p.blocks) {}
  __device__ int token(const PagedK& p) const { return grp * p.group + sub * BN; }
  __device__ int rows(const PagedK& p) const { return min(BN, p.group - sub * BN); }
  __device__ void step(const PagedK& p) {
    if (++sub == p.blocks) {
      sub = 0;
      ++grp;
    }
  }
};

template <bool WIN>
__device__ __forceinline__ int first_block(const Segment<WIN>& g) {
  return WIN && g.kb0 >= g.at.sb ? g.at.wb + (g.kb0 - g.at.sb) : g.kb0;
}

// From the tile's block kb to the next.
template <int BN, bool WIN>
__device__ __forceinline__ void next_block(const PagedP<WIN>& p, const Segment<WIN>& g, int kb,
                                           BlockPos<BN>& pos) {
  if (WIN && kb + 1 == g.at.sb)
    pos = BlockPos<BN>(p, g.at.wb);
  else
    pos.step(p);
}

// Page of a tile's count of them in the stream's list.
template <bool WIN>
__device__ __forceinline__ int page_index(const PagedP<WIN>& p, const Span<WIN>& at, int page) {
  if constexpr (WIN)
    return page >= at.cut >> p.page_log ? page + (at.shift >> p.page_log) : page;
  else
    return page;
}

// Where the tokens end that are there, as the tile counts them, in the block at `token`.
template <bool WIN>
__device__ __forceinline__ int held_to(const PagedP<WIN>& p, const Segment<WIN>& g, int token) {
  if constexpr (WIN)
    if (token < g.at.cut && g.at.cut > p.front) return min(p.front, g.st.len);
  return g.st.len - g.at.shift;
}

// What a row sees of a block, counted from its first token: the keys c < sinks, which are
// sinks, and low <= c < valid.
struct View {
  int sinks, low, valid;
};

// The lowest n bits of 32.
__device__ __forceinline__ unsigned low_bits(int n) {
  return n > 0 ? 0xffffffffu >> (32 - min(n, 32)) : 0u;
}

// Of a row whose keys end at `keys` and begin behind the sinks at `low`.
__device__ __forceinline__ View view_of(const PagedP<true>& p, const Segment<true>& g, int kb, int token,
                                        int keys, int low) {
  View v{0, low - g.at.shift - token, keys - g.at.shift - token};
  if (kb < g.at.sb) {
    v.sinks = min(p.sinks, keys) - token;
    if (!p.compact && p.turned) v.valid = 0;
    v.valid = max(v.valid, v.sinks);
  }
  return v;
}

// Whether the token u of the tile's count, in its block kb, is there as one of the sinks'
// pages, which their own queries score.
__device__ __forceinline__ bool among_sinks(const PagedP<true>& p, const Segment<true>& g, int kb,
                                            int u) {
  return p.compact ? u < g.at.cut : kb < g.at.sb;
}

// Whether the masks hide that token from all rows of the tile, whose first row's keys end at
// first_end and whose last row's at last_end: such a key may be NaN, and must not be
// multiplied by weights of 0. (Where a window is shorter than a block of the mask, keys
// before each block's window are hidden too.)
__device__ __forceinline__ bool tile_hides(const PagedP<true>& p, const Segment<true>& g, int kb, int u,
                                           int first_end, int last_end) {
  const bool sink = among_sinks(p, g, kb, u);
  const int j = sink ? u : u + g.at.shift;
  if (j >= last_end) return true;
  if (sink && j < p.sinks) return false;
  if (sink && p.turned) return true;
  int end = first_end;
  if (p.block > p.window) {
    const long long own =
        static_cast<long long>(p.by_mask(j + g.st.gone) + 1) * p.block - g.st.gone;
    end = max(end, static_cast<int>(min(own, static_cast<long long>(g.st.len))));
  }
  return j < first_key(p, end, g.st.gone);
}

// Whether it may hide one of the block's.
template <int BN>
__device__ __forceinline__ bool tile_hides_some(const PagedP<true>& p, const Segment<true>& g, int kb,
                                                int token, int tile_low, int last_end) {
  return token + BN > last_end - g.at.shift || p.block > p.window ||
         (kb < g.at.sb ? token + BN > p.sinks : token < tile_low - g.at.shift);
}

// Host side: the kernels' parameters for key blocks of bn tokens.
template <bool WIN>
PagedP<WIN> paged_params(const PagedAttnArgs& a, int bn, int dv) {
  const bool divides = bn % a.page_tokens == 0;
  const PartLayout at(dv);
  char* ws = PartLayout::base(a.workspace);
  PagedP<WIN> k;
  k.q_start = a.q_start;
  k.table = a.table;
  k.lens = a.lens;
  k.o = static_cast<__nv_bfloat16*>(a.o);
  k.part_o = reinterpret_cast<float*>(ws);
  k.part_ml = reinterpret_cast<float2*>(ws + at.ml);
  k.part_desc = reinterpret_cast<int4*>(ws + at.desc);
  k.total = a.total;
  k.heads = a.heads;
  k.seqs = a.seqs;
  k.pages = a.pages;
  k.page_tokens = a.page_tokens;
  k.max_pages = a.max_pages;
  k.block = a.causal_block;
  k.group = divides ? bn : a.page_tokens;
  k.blocks = (k.group + bn - 1) / bn;
  k.per_group = divides ? bn / a.page_tokens : 1;
  k.box_rows = divides ? a.page_tokens : bn;
  k.by_heads = div_by(k.heads);
  k.by_group = div_by(k.group);
  k.by_blocks = div_by(k.blocks);
  k.by_mask = div_by(k.block > 0 ? k.block : 1);
  k.scale_log2 = a.scale_log2;
  k.status = a.status;
  if constexpr (WIN) {
    k.dropped = a.dropped;
    k.window = a.window;
    k.sinks = a.sinks;
    k.front = sink_places(a.sinks, a.page_tokens);
    k.turned = a.q_sink != nullptr && a.sinks > 0;
    k.compact = divides;
    k.o_wide = aligned_to(a.o, 32);
    k.page_log = 0;
    while (divides && (1 << k.page_log) < a.page_tokens) ++k.page_log;
  }
  return k;
}

// CTAs that shared the work, cl of them a pair.
int launch_paged_join(const PagedK& k, int ctas, int cl, const PagedAttnArgs& a);
int launch_paged_decode(const PagedAttnArgs& a);
int launch_window_decode(const PagedAttnArgs& a);
int launch_window_teams(const PagedAttnArgs& a, int team, int teams);
int window_team_slots(int team);  // teams of 1, 2, 4 or 8 CTAs that run at a time

}  // namespace vmla
