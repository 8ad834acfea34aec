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

struct Stream {
  int q0, n, len;
};

__device__ __forceinline__ Stream stream_at(const PagedK& p, int s) {
  Stream t{p.q_start[s], p.q_start[s + 1], p.lens[s]};
  const int q1 = t.n;
  t.n = q1 - t.q0;
  if (t.q0 < 0 || q1 < t.q0 || q1 > p.total || t.len < 0 ||
      t.len > static_cast<long long>(p.max_pages) * p.page_tokens)
    t.n = 0;
  return t;
}

// Keys that the token at place a (it may be negative) of a stream of `held` tokens
// sees.
__device__ __forceinline__ int keys_seen(const PagedK& p, int a, int held) {
  if (a < 0) return 0;
  if (p.block == 0) return held;
  const long long end = static_cast<long long>(p.by_mask(a) + 1) * p.block;
  return end < held ? static_cast<int>(end) : held;
}

// Key blocks of row tile `tile` (TR rows) of a stream: what its last row, which
// sees most, needs; at least one, so that rows that see nothing are written.
template <int BN, int TR>
__device__ __forceinline__ int tile_blocks(const PagedK& p, int n, int len, int tile) {
  const int last = min(n * p.heads, (tile + 1) * TR) - 1;
  const int keys = keys_seen(p, len - n + p.by_heads(last), len);
  const int whole = p.by_group(keys), rest = keys - whole * p.group;
  return max(1, whole * p.blocks + (rest + BN - 1) / BN);
}

// Cost of a stream's row tiles in keys, as a straight line from the first to the
// last tile's keys (exact for a whole chunk and token by token, and within a
// mask block for others) plus kTileCost for loading Q and writing O: prefix sums
// in closed form, so a share's ends are found without walking the tiles. Four blocks:
// with two or eight the ragged and the drafted tokens' calls are 2 - 8 % slower.
template <int BN>
constexpr int kTileCost = 4 * BN;

struct Cost {
  long long first, slope;  // slope in 1/256 keys per tile
  int tiles;
  __device__ long long before(int t) const {  // of tiles 0 .. t-1
    return t * first + ((slope * (static_cast<long long>(t) * (t - 1) / 2)) >> 8);
  }
};

template <int BN, int TR>
__device__ __forceinline__ Cost cost_of(const PagedK& p, const Stream& st) {
  Cost c{0, 0, 0};
  if (st.n == 0) return c;
  const int rows = st.n * p.heads;
  c.tiles = (rows + TR - 1) / TR;
  const int k1 = keys_seen(p, st.len - 1, st.len);
  c.first = k1 + kTileCost<BN>;
  if (c.tiles > 1) {
    const int k0 = keys_seen(p, st.len - st.n + p.by_heads(TR - 1), st.len);
    if (c.tiles <= 4096) {  // the products stay below 2^63
      c.first = k0 + kTileCost<BN>;
      c.slope = static_cast<long long>(__fdividef((k1 - k0) * 256.f, c.tiles - 1.f));
    } else {
      c.first = (static_cast<long long>(k0) + k1) / 2 + kTileCost<BN>;
    }
  }
  return c;
}

struct Place {
  int s, tile, off;  // stream, row tile, key block
  int all;           // the tile's key blocks
  Stream st;
};

// The shares' ends: place of share id's first block and of the one after its
// last. Every thread of the block calls it; scratch: 8 long longs and out: two
// Places in shared memory. Three warps look for each end, all streams among their
// 96 threads: one search's latency, not two, is part of every call. With more slots
// than that, idle ones included, a thread walks several of them in turn: one token of
// 16 streams on 2,000 keys takes 13.9 us with 16 slots, 21 with 96, 115 with 1,024 and
// 908 with 8,192. Returns the cost of a share.
template <int BN, int TR>
__device__ __forceinline__ long long find_share(const PagedK& p, int id, int groups,
                                                long long* scratch, Place* out) {
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const int e = warp / 3;  // which end; the other warps only wait
  const int per = (p.seqs + 95) / 96;
  const int s0 = (threadIdx.x - e * 96) * per;
  long long mine = 0;
  Stream st{0, 0, 0};
  Cost c{0, 0, 0};
  if (e < 2)
    for (int k = 0; k < per; ++k)
      if (s0 + k < p.seqs) {
        st = stream_at(p, s0 + k);
        c = cost_of<BN, TR>(p, st);
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
          st = stream_at(p, s);
          c = cost_of<BN, TR>(p, st);
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
        const int blocks = tile_blocks<BN, TR>(p, st.n, st.len, lo);
        const int off = static_cast<int>(
            static_cast<float>(rem - at) *
            __fdividef(static_cast<float>(blocks), static_cast<float>(c.before(lo + 1) - at)));
        out[e] = Place{s, lo, min(off, blocks - 1), blocks, st};
      }
    }
  }
  __syncthreads();
  return active > 0 ? static_cast<long long>(__fdividef(static_cast<float>(total), active)) : 0;
}

// Walks a share segment by segment: a segment is a run of key blocks of one row
// tile. Every role of the CTA walks it for itself.
struct Segment {
  Stream st;
  int s, tile;
  int kb0, kb1, all;   // key blocks [kb0, kb1) of the tile's `all`
};

template <int BN, int TR>
struct Walk {
  const PagedK& p;
  Stream st;
  int s, tile, off, all;  // all < 0: not known yet
  int end_s, end_tile, end_off;
  __device__ Walk(const PagedK& k, const Place* ends) : p(k) {
    st = ends[0].st;  // the first segment needs no arithmetic: the search had it all
    s = ends[0].s;
    tile = ends[0].tile;
    off = ends[0].off;
    all = ends[0].all;
    end_s = ends[1].s;
    end_tile = ends[1].tile;
    end_off = ends[1].off;
  }
  __device__ bool next(Segment& g) {
    if (s >= p.seqs) return false;
    if (all < 0) {
      while (tile * TR >= st.n * p.heads) {  // a stream with new tokens
        if (++s >= p.seqs) return false;
        st = stream_at(p, s);
        tile = 0;
      }
      all = tile_blocks<BN, TR>(p, st.n, st.len, tile);
    }
    const bool last = s == end_s && tile == end_tile;
    if (s > end_s || (s == end_s && tile > end_tile) || (last && off >= end_off)) return false;
    g.st = st;
    g.s = s;
    g.tile = tile;
    g.kb0 = off;
    g.kb1 = last ? end_off : all;
    g.all = all;
    off = 0;
    all = -1;
    ++tile;
    return true;
  }
};

// Place of key block kb: its first token, and the rows of its group from there.
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

// Host side: the kernels' parameters for key blocks of bn tokens.
inline PagedK paged_params(const PagedAttnArgs& a, int bn, int dv) {
  const bool divides = bn % a.page_tokens == 0;
  const PartLayout at(dv);
  char* ws = PartLayout::base(a.workspace);
  PagedK k;
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
  return k;
}

int launch_paged_join(const PagedK& k, int ctas, const PagedAttnArgs& a);
int launch_paged_decode(const PagedAttnArgs& a);

}  // namespace vmla
