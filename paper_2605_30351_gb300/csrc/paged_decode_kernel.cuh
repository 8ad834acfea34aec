// Attention over a paged latent cache for streams of few rows (Eq. score; App. E):
// a decoding step, where a stream has up to 16 (token, head) rows.
//
// Each key is read once for 16 rows, so the step is bound by reading the cache (at
// d_c = 192, d_r = 32: 448 bytes and 13.3 kFLOP a key, 30 FLOP a byte where the card does
// 280 a byte at its measured rates, mma.sync a fraction of that). The tensor-memory path pads
// 16 rows to 128 and passes every block through four warps in turn (scores,
// softmax, weights, output); here each of eight warps takes 16 keys of a block of
// 128 through all steps by itself, with mma.sync tiles of 16 rows, and waits for no
// other warp until the stream's keys are done:
//     K, C                                 asynchronous copies of 16 bytes into the
//                                          warp's own ring of 16-key stages, zeros
//                                          where a row holds no token
//     S = Q K^T (16 x 16, K = d_c + d_r)   Q fragments in registers (shared memory
//                                          at d_c = 256, where O fills them)
//     P = exp2(S * log2(e)/sqrt(d_h) - m)  the warp's own running maximum and sum
//     O += P C                             P's accumulator layout is the next A
//                                          operand's; C read transposed (ldmatrix).
//                                          P is rounded to bf16, the type of C, as the
//                                          mma takes both operands of one type; its sum
//                                          is that of the unrounded weights, in fp32
// The warps' O, maxima and sums are added up in shared memory at the end of a
// segment. Shares, partial rows and their join are those of paged_attn.cu.
//
// Pages that do not divide a block of 128 keys are blocks of their own: with 24 tokens a
// page two warps of eight have keys, and the last of them half a tile (64 streams on 8,000
// keys 140 us, with 16 or 32 tokens a page 53 and 50).
//
// Measured on the GPU at d_c = 192, d_r = 32, 12 heads: one token on 777 keys 9.2 us and on
// 32,760 keys 13.4 us (latency: the share search, the first keys, the join); 64
// streams of up to 32,760 keys 78.0 us (416 MB, 5.3 TB/s; 76 us of it this kernel,
// DRAM at 70 % of its peak over the kernel's start and end). The tensor-memory path
// on the same calls: 13.3, 18.0 and 79.4 us, and with pages of 16 tokens, whose
// copies are 2 KB boxes there, 102 us instead of 84.5.
//
// With a sliding window (WIN) a warp leaves out 16 keys that no row of the tile sees, and the
// sinks' keys are scored by their own q_r (fragments loaded again where a warp passes from
// sinks to window). 64 streams, one sink frame of 1,560 and a window of 9,360 tokens (12 heads,
// d_c = 192): 57.7 us, 229 MB, exactly the bytes needed (ncu: 229.1 MB read), 4.0 TB/s over the
// call and 5.8 between start and end.
// Teams (TEAM): where a window bounds the keys of a tile, a cluster of 1 to 8 CTAs takes whole
// tiles, each CTA a part of their blocks, and the CTAs send their rows (maximum, sum, O) to one
// another's shared memory, where each joins its share of the 16 rows, parts in order: no share
// search, no partial rows in the workspace, no second launch. One token on a window of 512 and
// 4 sinks 8.7 us, by shares 10.6. What is left is latency: row starts, the page table, keys,
// the warps' sums, the cluster's barrier, about a microsecond each.

#pragma once

#include "internal.h"
#include "paged_attn.cuh"
#include "ptx_sm103.cuh"

namespace vmla {
namespace {

constexpr int kWarps = 8;
constexpr int kDecodeThreads = 32 * kWarps;
constexpr int kRows = 16;                     // rows of a tile
constexpr int kBN = 16 * kWarps;              // keys of a block
constexpr float kMoveLog2 = 8.0f;             // how far a maximum lags behind

template <int DC, int DR, bool WIN, bool TEAM>
struct DecodeShape {
  static constexpr int DK = DC + DR;
  static constexpr int kTileBytes = 16 * DK * 2;  // a warp's stage of 16 keys:
  static constexpr int kCBox = 16 * 128;          // [16 x 64 columns] of c each,
  static constexpr int kKrOff = DC * 16 * 2;      // then the d_r columns
  static constexpr int kKrRow = DR * 2;
  // Q's rows, with a window the sinks' q_r behind them
  static constexpr int kQStride = (WIN ? DK + DR : DK) * 2 + 16;  // bytes; rows in different banks
  static constexpr int kQBytes = kRows * kQStride;
  // The warps' results at the end of a segment, floats per row: 32 columns at a time in two
  // buffers, or in a team, whose calls are short, all at once in the place of the ring (one
  // wait instead of six: one token of 38 streams 9.8 -> 9.3 us; but the decoding step of 64
  // long streams 60.6 -> 62.3).
  static constexpr int kRedStride = TEAM ? DC + 8 : 32 + 8;
  static constexpr int kRedBytes = TEAM ? 0 : 2 * kWarps * kRows * kRedStride * 4;
  static constexpr int kTeamBytes = TEAM ? kRows * (DC * 4 + 8) : 0;
  static constexpr int kMlBytes = kWarps * kRows * 8;
  static constexpr int kRest = 1024 + kQBytes + kRedBytes + kMlBytes + kTeamBytes + 192;
  static constexpr int kFit = (232448 - kRest) / (kTileBytes * kWarps);
  static constexpr int kStages = kFit > 4 ? 4 : kFit;
  static constexpr int kSmemBytes = kRest + kTileBytes * kWarps * kStages;
  static constexpr bool kQRegs = DC <= 192;
  static_assert(kStages >= 2 && kQBytes % 16 == 0, "two stages must fit");
  static_assert(!TEAM || kRows * kRedStride * 4 <= kTileBytes * kStages,
                "the warps' results fit in the ring");
  static_assert(64 + 2 * sizeof(Place<WIN>) <= 192, "the search's sums and the share's ends fit");
};

__device__ __forceinline__ void ldm4(uint32_t (&r)[4], uint32_t addr) {
  asm volatile("ldmatrix.sync.aligned.m8n8.x4.shared.b16 {%0, %1, %2, %3}, [%4];"
               : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3])
               : "r"(addr)
               : "memory");
}
__device__ __forceinline__ void ldm4t(uint32_t (&r)[4], uint32_t addr) {
  asm volatile("ldmatrix.sync.aligned.m8n8.x4.trans.shared.b16 {%0, %1, %2, %3}, [%4];"
               : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3])
               : "r"(addr)
               : "memory");
}
__device__ __forceinline__ void mma16816(float (&d)[4], const uint32_t (&a)[4], uint32_t b0,
                                         uint32_t b1) {
  asm volatile(
      "mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, "
      "{%8, %9}, {%0, %1, %2, %3};"
      : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
      : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}
// 16 bytes to shared memory, of which `bytes` (16 or 0) are read and the rest zeros.
__device__ __forceinline__ void copy16(uint32_t dst, const void* src, int bytes) {
  asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(dst), "l"(src), "r"(bytes)
               : "memory");
}

template <int DC, int DR, bool WIN, bool TEAM>
__global__ void __launch_bounds__(kDecodeThreads, 1)
    paged_decode_kernel(const uint8_t* c, const uint8_t* kr, const __nv_bfloat16* q_c,
                        const __nv_bfloat16* q_r, const __nv_bfloat16* q_sink, const PagedP<WIN> p) {
  using S = DecodeShape<DC, DR, WIN, TEAM>;
  constexpr int NST = S::kStages, kSteps = S::DK / 16;
  extern __shared__ uint8_t smem_raw[];
  uint8_t* sKV = align_smem_1024(smem_raw);
  uint8_t* sQ = sKV + NST * kWarps * S::kTileBytes;
  float* red = reinterpret_cast<float*>(TEAM ? sKV : sQ + S::kQBytes);  // [warps][16][kRedStride]
  float2* warp_ml = reinterpret_cast<float2*>(sQ + S::kQBytes + S::kRedBytes);
  // of a team: [its CTAs][this one's rows] (maximum, sum), then the rows
  float2* team_ml = warp_ml + kWarps * kRows;
  float* team_o = reinterpret_cast<float*>(team_ml + (TEAM ? kRows : 0));
  long long* scratch = reinterpret_cast<long long*>(team_o + (TEAM ? kRows * DC : 0));  // [8]
  Place<WIN>* ends = reinterpret_cast<Place<WIN>*>(scratch + 8);                         // [2]

  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  grid_dep_sync();
  // one block looks at the metadata; with a window while its first keys are on their way
  bool checked = blockIdx.x != 0;
  auto check = [&]() {
    if (!checked) check_streams<WIN>(p, threadIdx.x, kDecodeThreads);
    checked = true;
  };
  if constexpr (!WIN) check();
  // What a CTA computes: a share of all tiles' blocks, or as one of a team of CTAs (a
  // cluster), which takes whole streams in turn, its part of each of their tiles.
  const int team = TEAM ? static_cast<int>(cluster_nctarank()) : 1;
  const int member = TEAM ? static_cast<int>(cluster_ctarank()) : 0;
  if constexpr (TEAM) {
    cluster_arrive_release();  // a wait before sending: the others run, and have read
  } else {
    if (threadIdx.x < 2) p.part_desc[2 * blockIdx.x + threadIdx.x] = make_int4(0, 0, 0, 0);
    find_share<kBN, kRows, WIN>(p, blockIdx.x, gridDim.x, scratch, ends);
  }
  Segment<WIN> g;
  auto walk = [&]() {
    if constexpr (TEAM) {
      const int id = blockIdx.x / team;
      const Stream<true> first = id < p.seqs ? stream_at<true>(p, id) : Stream<true>{};
      bool further = false;  // tiles that are not a stream's first
      for (int k = threadIdx.x; k < p.seqs; k += kDecodeThreads)
        further |= static_cast<long long>(p.q_start[k + 1] - p.q_start[k]) * p.heads > kRows;
      return TeamWalk<kBN, kRows>(p, id, gridDim.x / team, first, __syncthreads_or(further));
    } else {
      return Walk<kBN, kRows, WIN>(p, ends);
    }
  }();
  auto next_segment = [&]() {
    if (!walk.next(g)) return false;
    if constexpr (TEAM) {
      g.kb0 = static_cast<int>(static_cast<long long>(g.at.all) * member / team);
      g.kb1 = static_cast<int>(static_cast<long long>(g.at.all) * (member + 1) / team);
    }
    return true;
  };
  const int ra = lane >> 2, rb = ra + 8;  // the lane's two rows
  const int cq = 2 * (lane & 3);          // and the first of its two columns in a tile of 8
  // ldmatrix addresses: Q, keys (two tiles of 8 keys x 16 values), values transposed
  const uint32_t q_at = smem_u32(sQ) + (lane & 15) * S::kQStride + (lane >> 4) * 16;
  const int k_row = (lane & 7) + ((lane >> 4) & 1) * 8, k_half = (lane >> 3) & 1;
  const int v_row = (lane & 7) + ((lane >> 3) & 1) * 8, v_half = lane >> 4;
  const uint32_t ring = smem_u32(sKV) + warp * NST * S::kTileBytes;
  // This warp's 16 keys of a block lie in one page, or with pages of 8 tokens in
  // two: whole pages up to 16 of them, or a run inside one.
  const bool small = p.per_group > 1 || p.group == kBN;  // pages divide a block
  const int page_step = p.page_tokens < 16 && small ? 1 : 0;
  const int page_at = small ? 16 * warp / p.page_tokens : 0;
  const int off_at = small ? 16 * warp - page_at * p.page_tokens : 16 * warp;
  bool any = false;
  while (next_segment()) {
    any = true;
    const int rows = g.st.n * p.heads, row0 = g.tile * kRows;
    const int n_rows = min(kRows, rows - row0);
    const size_t grow = static_cast<size_t>(g.st.q0) * p.heads + row0;
    bool own_qr = false;  // the sinks' queries are needed
    if constexpr (WIN) own_qr = p.turned && g.kb0 < g.at.sb;
    auto keys_of = [&](int r) {
      return r < n_rows
                 ? keys_seen<WIN>(p, g.st.len - g.st.n + p.by_heads(row0 + r), g.st)
                 : 0;
    };
    const int keys_a = keys_of(ra), keys_b = keys_of(rb);
    int low_a = 0, low_b = 0, first_end = 0, last_end = 0, first_low = 0;
    if constexpr (WIN) {
      low_a = first_key(p, keys_a, g.st.gone);
      low_b = first_key(p, keys_b, g.st.gone);
      first_end = keys_of(0);
      last_end = keys_of(n_rows - 1);
      first_low = first_key(p, first_end, g.st.gone);
    }

    // The ring: block kb0 + i goes to stage i % NST, NST - 1 blocks ahead of the one
    // that is computed. The pages of the next block to fetch are looked up one
    // block ahead of that.
    const int n_blocks = g.kb1 - g.kb0;
    const int* table = p.table + static_cast<size_t>(g.s) * p.max_pages;
    BlockPos<kBN> ahead(p, first_block(g));
    int page_a = -1, page_b = -1;
    // tokens among the warp's 16 keys of block i; with a window none where no row of the
    // tile sees one of them
    auto held = [&](const BlockPos<kBN>& at, int i) {
      const int token = at.token(p) + 16 * warp;
      if constexpr (WIN) {
        const bool sinks = among_sinks(p, g, g.kb0 + i, token);
        const int from = sinks ? token : token + g.at.shift;
        if (from >= last_end ||
            !((sinks && from < p.sinks) || (!(sinks && p.turned) && from + 16 > first_low)))
          return 0;
        return min(at.rows(p) - 16 * warp, held_to(p, g, token) - token);
      }
      return min(at.rows(p) - 16 * warp, g.st.len - token);
    };
    auto look_up = [&](int i) {
      if (i < n_blocks && held(ahead, i) > 0) {
        const int at = ahead.grp * p.per_group + page_at;
        page_a = table[page_index(p, g.at, at)];
        page_b = page_step && held(ahead, i) > 8 ? table[page_index(p, g.at, at + 1)] : page_a;
      }
    };
    auto fetch = [&](int i) {
      const int n = i < n_blocks ? held(ahead, i) : 0;
      if (n > 0) {
        // keys that no row of the tile sees come as zeros: they may be NaN
        unsigned shown = 0xffffu;
        if constexpr (WIN) {
          const int token = ahead.token(p) + 16 * warp;
          if (g.kb0 + i < g.at.sb || token + 16 > last_end - g.at.shift ||
              token < first_low - g.at.shift || p.block > p.window)
            shown = __ballot_sync(0xffffffffu, lane < 16 && !tile_hides(p, g, g.kb0 + i, token + lane,
                                                                        first_end, last_end));
        }
        if (page_a < 0 || page_a >= p.pages || page_b < 0 || page_b >= p.pages)
          record_status(p.status, MLA_ERR_RANGE);
        const uint32_t dst = ring + (i % NST) * S::kTileBytes;
        const int off = ahead.sub * kBN + off_at;
#pragma unroll
        for (int rg = 0; rg < 4; ++rg) {  // 4 rows x 128 bytes of c at a time
          const int row = 4 * rg + (lane >> 3), pc = lane & 7;
          const int page = row < 8 ? page_a : page_b;
          const bool in = row < n && page >= 0 && page < p.pages && (!WIN || (shown >> row & 1));
          const size_t at = in ? static_cast<size_t>(page) * p.page_tokens + off + row -
                                     (page_step && row >= 8 ? 8 : 0)
                               : 0;
          const uint8_t* src = c + at * (DC * 2) + pc * 16;
#pragma unroll
          for (int cb = 0; cb < DC / 64; ++cb)
            copy16(dst + cb * S::kCBox + row * 128 + ((pc ^ (row & 7)) * 16), src + cb * 128,
                   in ? 16 : 0);
        }
        constexpr int kPr = DR / 8, kAtOnce = 32 / kPr;  // pieces of a key row, rows at a time
#pragma unroll
        for (int rg = 0; rg < 16 / kAtOnce; ++rg) {
          const int row = kAtOnce * rg + lane / kPr, pc = lane % kPr;
          const int page = row < 8 ? page_a : page_b;
          const bool in = row < n && page >= 0 && page < p.pages && (!WIN || (shown >> row & 1));
          const size_t at = in ? static_cast<size_t>(page) * p.page_tokens + off + row -
                                     (page_step && row >= 8 ? 8 : 0)
                               : 0;
          const int sw = DR == 32 ? (row >> 1) & 3 : row & 7;
          copy16(dst + S::kKrOff + row * S::kKrRow + ((pc ^ sw) * 16),
                 kr + at * (DR * 2) + pc * 16, in ? 16 : 0);
        }
      }
      asm volatile("cp.async.commit_group;" ::: "memory");
      next_block<kBN>(p, g, g.kb0 + i, ahead);
      look_up(i + 1);
    };
    look_up(0);
    // Q's rows (zeros where the tile has none) are on their way while the page is looked up
    constexpr int kPc = DC / 8, kPr = DR / 8;  // 16-byte pieces of a row
    constexpr int kPq = WIN ? kPc + 2 * kPr : kPc + kPr;
    for (int i = threadIdx.x; i < kRows * kPq; i += kDecodeThreads) {
      const int r = i / kPq, pc = i - r * kPq;
      if (WIN && pc >= kPc + kPr && !own_qr) continue;
      const size_t row = grow + (r < n_rows ? r : 0);
      const __nv_bfloat16* src = pc < kPc ? q_c + row * DC + pc * 8
                                          : (pc < kPc + kPr ? q_r + row * DR + (pc - kPc) * 8
                                                            : q_sink + row * DR + (pc - kPc - kPr) * 8);
      copy16(smem_u32(sQ) + r * S::kQStride + pc * 16, src, r < n_rows ? 16 : 0);
    }
    asm volatile("cp.async.commit_group;" ::: "memory");
#pragma unroll 1
    for (int i = 0; i < NST - 1; ++i) fetch(i);
    if constexpr (WIN) check();
    asm volatile("cp.async.wait_group %0;" ::"n"(NST - 1) : "memory");
    __syncthreads();
    uint32_t q[S::kQRegs ? kSteps : 1][4];
    if constexpr (S::kQRegs) {
#pragma unroll
      for (int k = 0; k < kSteps; ++k)
        ldm4(q[k], q_at + k * 32);
    }
    float o[DC / 8][4];
#pragma unroll
    for (int i = 0; i < DC / 8; ++i)
#pragma unroll
      for (int c = 0; c < 4; ++c) o[i][c] = 0.f;
    float m_a = -INFINITY, m_b = -INFINITY, l_a = 0.f, l_b = 0.f;

    BlockPos<kBN> pos(p, first_block(g));
    bool q_is_sinks = false;
#pragma unroll 1
    for (int i = 0; i < n_blocks; ++i, next_block<kBN>(p, g, g.kb0 + i - 1, pos)) {
      fetch(i + NST - 1);
      const int token = pos.token(p) + 16 * warp, room = pos.rows(p) - 16 * warp;
      bool sinks_q = false;  // the warp's keys are scored by the sinks' own q_r
      if constexpr (WIN) {
        sinks_q = own_qr && among_sinks(p, g, g.kb0 + i, token);
        if (S::kQRegs && sinks_q != q_is_sinks) {
#pragma unroll
          for (int k = DC / 16; k < kSteps; ++k)
            ldm4(q[k], q_at + k * 32 + (sinks_q ? DR * 2 : 0));
          q_is_sinks = sinks_q;
        }
      }
      asm volatile("cp.async.wait_group %0;" ::"n"(NST - 1) : "memory");
      __syncwarp();
      if (held(pos, i) > 0) {
        const uint32_t ka = ring + (i % NST) * S::kTileBytes;
        float s[2][4];  // two tiles of 8 keys
#pragma unroll
        for (int t = 0; t < 2; ++t)
#pragma unroll
          for (int c = 0; c < 4; ++c) s[t][c] = 0.f;
#pragma unroll
        for (int k = 0; k < kSteps; ++k) {
          uint32_t b[4];
          if (k < DC / 16) {
            const int pc = 2 * (k & 3) + k_half;
            ldm4(b, ka + (k >> 2) * S::kCBox + k_row * 128 + ((pc ^ (k_row & 7)) * 16));
          } else {
            const int pc = 2 * (k - DC / 16) + k_half;
            const int sw = DR == 32 ? (k_row >> 1) & 3 : k_row & 7;
            ldm4(b, ka + S::kKrOff + k_row * S::kKrRow + ((pc ^ sw) * 16));
          }
          if constexpr (S::kQRegs) {
            mma16816(s[0], q[k], b[0], b[1]);
            mma16816(s[1], q[k], b[2], b[3]);
          } else {
            ldm4(q[0], q_at + k * 32 + (k >= DC / 16 && sinks_q ? DR * 2 : 0));
            mma16816(s[0], q[0], b[0], b[1]);
            mma16816(s[1], q[0], b[2], b[3]);
          }
        }
        if constexpr (WIN) {
          const View a = view_of(p, g, g.kb0 + i, token, keys_a, low_a);
          const View b = view_of(p, g, g.kb0 + i, token, keys_b, low_b);
          const int lim_a = min(room, a.valid), lim_b = min(room, b.valid);
#pragma unroll
          for (int t = 0; t < 2; ++t)
#pragma unroll
            for (int c = 0; c < 2; ++c) {
              const int key = 8 * t + cq + c;
              if (key >= lim_a || (key < a.low && key >= a.sinks)) s[t][c] = -INFINITY;
              if (key >= lim_b || (key < b.low && key >= b.sinks)) s[t][2 + c] = -INFINITY;
            }
        } else {
          const int lim_a = min(room, keys_a - token), lim_b = min(room, keys_b - token);
#pragma unroll
          for (int t = 0; t < 2; ++t)
#pragma unroll
            for (int c = 0; c < 2; ++c) {
              const int key = 8 * t + cq + c;
              if (key >= lim_a) s[t][c] = -INFINITY;
              if (key >= lim_b) s[t][2 + c] = -INFINITY;
            }
        }
        float x_a = fmaxf(fmaxf(s[0][0], s[0][1]), fmaxf(s[1][0], s[1][1]));
        float x_b = fmaxf(fmaxf(s[0][2], s[0][3]), fmaxf(s[1][2], s[1][3]));
#pragma unroll
        for (int d = 1; d < 4; d <<= 1) {
          x_a = fmaxf(x_a, __shfl_xor_sync(0xffffffffu, x_a, d));
          x_b = fmaxf(x_b, __shfl_xor_sync(0xffffffffu, x_b, d));
        }
        x_a *= p.scale_log2;
        x_b *= p.scale_log2;
        // The running maximum moves when a key exceeds it by more than 2^8 (weights
        // up to 256 are harmless in bf16 and fp32), or with the first key seen.
        const bool up_a = x_a > m_a + kMoveLog2 || (m_a == -INFINITY && x_a > m_a);
        const bool up_b = x_b > m_b + kMoveLog2 || (m_b == -INFINITY && x_b > m_b);
        if (__any_sync(0xffffffffu, up_a || up_b)) {
          const float f_a = up_a ? ex2_approx(m_a - x_a) : 1.f;
          const float f_b = up_b ? ex2_approx(m_b - x_b) : 1.f;
          if (up_a) m_a = x_a;
          if (up_b) m_b = x_b;
          l_a *= f_a;
          l_b *= f_b;
#pragma unroll
          for (int i = 0; i < DC / 8; ++i) {
            o[i][0] *= f_a;
            o[i][1] *= f_a;
            o[i][2] *= f_b;
            o[i][3] *= f_b;
          }
        }
        const float n_a = m_a == -INFINITY ? 0.f : -m_a, n_b = m_b == -INFINITY ? 0.f : -m_b;
        uint32_t w[4];  // P as the A operand: rows a, b of keys 0..7, then of 8..15
#pragma unroll
        for (int i = 0; i < 2; ++i) {
          const float a0 = ex2_approx(fmaf(s[i][0], p.scale_log2, n_a));
          const float a1 = ex2_approx(fmaf(s[i][1], p.scale_log2, n_a));
          const float b0 = ex2_approx(fmaf(s[i][2], p.scale_log2, n_b));
          const float b1 = ex2_approx(fmaf(s[i][3], p.scale_log2, n_b));
          l_a += a0 + a1;
          l_b += b0 + b1;
          w[2 * i] = pack_bf16x2(a0, a1);
          w[2 * i + 1] = pack_bf16x2(b0, b1);
        }
#pragma unroll
        for (int c = 0; c < DC / 16; ++c) {
          uint32_t b[4];
          const int pc = 2 * (c & 3) + v_half;
          ldm4t(b, ka + (c >> 2) * S::kCBox + v_row * 128 + ((pc ^ (v_row & 7)) * 16));
          mma16816(o[2 * c], w, b[0], b[1]);
          mma16816(o[2 * c + 1], w, b[2], b[3]);
        }
      }
      __syncwarp();  // the stage is the next copy's to overwrite
    }

    // The warps' results together, and out: finished rows as bf16, a cut tile's as
    // fp32 partial rows.
#pragma unroll
    for (int d = 1; d < 4; d <<= 1) {
      l_a += __shfl_xor_sync(0xffffffffu, l_a, d);
      l_b += __shfl_xor_sync(0xffffffffu, l_b, d);
    }
    if ((lane & 3) == 0) {
      warp_ml[warp * kRows + ra] = make_float2(m_a, l_a);
      warp_ml[warp * kRows + rb] = make_float2(m_b, l_b);
    }
    __syncthreads();
    const bool whole = TEAM ? team == 1 : g.kb0 == 0 && g.kb1 == g.at.all;
    const int slot = 2 * blockIdx.x + (g.kb0 == 0 ? 1 : 0);
    // row r over all warps: maximum, sum
    auto total_of = [&](int r) {
      float m = -INFINITY, l = 0.f;
#pragma unroll
      for (int w = 0; w < kWarps; ++w) m = fmaxf(m, warp_ml[w * kRows + r].x);
      const float ref = m == -INFINITY ? 0.f : m;
#pragma unroll
      for (int w = 0; w < kWarps; ++w) {
        const float2 ml = warp_ml[w * kRows + r];
        l += ex2_approx(ml.x - ref) * ml.y;
      }
      return make_float2(m, l);
    };
    const float2 t_a = total_of(ra), t_b = total_of(rb);
    auto factor = [&](float m, float2 t) {
      // a row that saw no key is 0; a NaN sum stays one
      const float f = ex2_approx(m - (t.x == -INFINITY ? 0.f : t.x));
      return whole ? (t.y == 0.f ? 0.f : f / t.y) : f;
    };
    const float f_a = factor(m_a, t_a), f_b = factor(m_b, t_b);
    const int out_r = threadIdx.x >> 4, out_c = 2 * (threadIdx.x & 15);
    const int to_rows = kRows / team;  // rows that each of a team joins
    uint32_t to_o = 0;
    if constexpr (TEAM)
      if (team > 1) {
        cluster_wait_acquire();
        to_o = dsmem_addr(smem_u32(team_o + ((member * to_rows + out_r % to_rows) * DC + out_c)),
                          out_r / to_rows);
      }
    // the warps' sum of the thread's row and two columns from 32 c on
    auto put = [&](const float* buf, int c, int col) {
      float2 sum = make_float2(0.f, 0.f);
#pragma unroll
      for (int w = 0; w < kWarps; ++w) {
        const float2 v = *reinterpret_cast<const float2*>(
            buf + (w * kRows + out_r) * S::kRedStride + col + out_c);
        sum.x += v.x;
        sum.y += v.y;
      }
      if (out_r >= n_rows) return;
      if (whole)
        *reinterpret_cast<uint32_t*>(p.o + (grow + out_r) * DC + 32 * c + out_c) =
            pack_bf16x2(sum.x, sum.y);
      else if constexpr (TEAM)
        dsmem_st_f32x2(to_o + 32 * c * 4, sum.x, sum.y);
      else
        *reinterpret_cast<float2*>(p.part_o + (static_cast<size_t>(slot) * kBM + out_r) * DC +
                                   32 * c + out_c) = sum;
    };
    auto lay = [&](float* buf, int i, int col) {  // this warp's columns 8 i .. 8 i + 7
      float* at = buf + (warp * kRows + ra) * S::kRedStride + col + cq;
      const float(&v)[4] = o[i];
      *reinterpret_cast<float2*>(at) = make_float2(v[0] * f_a, v[1] * f_a);
      *reinterpret_cast<float2*>(at + 8 * S::kRedStride) = make_float2(v[2] * f_b, v[3] * f_b);
    };
    if constexpr (TEAM) {  // the ring is free: every warp's loop has ended
#pragma unroll
      for (int i = 0; i < DC / 8; ++i) lay(red, i, 8 * i);
      __syncthreads();
#pragma unroll
      for (int c = 0; c < DC / 32; ++c) put(red, c, 32 * c);
    } else {
#pragma unroll
      for (int c = 0; c < DC / 32; ++c) {
        float* buf = red + (c & 1) * kWarps * kRows * S::kRedStride;
#pragma unroll
        for (int i = 0; i < 4; ++i) lay(buf, 4 * c + i, 8 * i);
        __syncthreads();
        put(buf, c, 0);
      }
    }
    if (!whole && threadIdx.x < n_rows) {
      float2 t = total_of(threadIdx.x);
      const int keys = keys_of(threadIdx.x);
      bool sees = keys > BlockPos<kBN>(p, first_block(g)).token(p);
      if constexpr (WIN) {  // one of the segment's keys
        const int low = first_key(p, keys, g.st.gone);
        sees = false;
        BlockPos<kBN> at(p, first_block(g));
        for (int kb = g.kb0; kb < g.kb1 && !sees; ++kb, next_block<kBN>(p, g, kb - 1, at)) {
          const View v = view_of(p, g, kb, at.token(p), keys, low);
          sees = v.sinks > 0 || max(v.low, 0) < min(at.rows(p), v.valid);
        }
      }
      if (sees) t.x = fmaxf(t.x, kLowest);
      if constexpr (TEAM) {
        const int r = threadIdx.x;
        dsmem_st_f32x2(dsmem_addr(smem_u32(team_ml + member * to_rows + r % to_rows), r / to_rows),
                       t.x, t.y);
      } else {
        p.part_ml[slot * kBM + threadIdx.x] = t;
      }
    }
    if constexpr (!TEAM)
      if (!whole && threadIdx.x == 0)
        p.part_desc[slot] = make_int4(static_cast<int>(grow), n_rows,
                                      kPartHeld | (g.kb1 == g.at.all ? kPartEnds : 0), 2);
    if constexpr (TEAM)
      if (team > 1) {
        // every CTA joins its rows, parts in their order
        __syncwarp();
        cluster_sync();
        for (int i = threadIdx.x; i < to_rows * (DC / 2); i += kDecodeThreads) {
          const int r = i / (DC / 2), col = 2 * (i - r * (DC / 2)), row = member * to_rows + r;
          if (row >= n_rows) continue;
          float m = -INFINITY;
          for (int k = 0; k < team; ++k) m = fmaxf(m, team_ml[k * to_rows + r].x);
          const float ref = m == -INFINITY ? 0.f : m;
          float l = 0.f, x = 0.f, y = 0.f;
          for (int k = 0; k < team; ++k) {
            const float2 ml = team_ml[k * to_rows + r];
            if (ml.x == -INFINITY) continue;  // the part has no key that the row sees
            const float2 v = *reinterpret_cast<const float2*>(team_o + (k * to_rows + r) * DC + col);
            const float w = ex2_approx(ml.x - ref);
            l += w * ml.y;
            x += w * v.x;
            y += w * v.y;
          }
          const float f = l == 0.f ? 0.f : 1.f / l;
          *reinterpret_cast<uint32_t*>(p.o + (grow + row) * DC + col) = pack_bf16x2(x * f, y * f);
        }
        cluster_arrive_release();
      }
    __syncthreads();  // sQ, the sums and the buffers are the next segment's
  }
  if constexpr (WIN) check();
  if constexpr (TEAM) {
    cluster_wait_acquire();
  } else {
    if (!any && threadIdx.x == 0)
      p.part_desc[2 * blockIdx.x] = make_int4(0, 0, kPartEmpty, 0);
  }
}

template <int DC, int DR, bool WIN>
int launch_decode(const PagedAttnArgs& a) {
  using S = DecodeShape<DC, DR, WIN, false>;
  const PagedP<WIN> k = paged_params<WIN>(a, kBN, DC);
  auto kern = paged_decode_kernel<DC, DR, WIN, false>;
  static PerDevice known;  // one CTA per SM, asked once
  std::atomic<int>* cell = known.cell();
  if (!cell) return MLA_ERR_CUDA;
  int ctas = cell->load();
  if (ctas == 0) {
    int dev = 0, sms = 0;
    cudaError_t e =
        cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, S::kSmemBytes);
    if (e == cudaSuccess) e = cudaGetDevice(&dev);
    if (e == cudaSuccess)
      e = cudaDeviceGetAttribute(&sms, cudaDevAttrMultiProcessorCount, dev);
    if (e == cudaSuccess && sms < 1) e = cudaErrorInvalidDevice;
    if (e != cudaSuccess) {
      (void)cudaGetLastError();
      set_last_cuda_error(e);
      return MLA_ERR_CUDA;
    }
    ctas = sms < kMaxCtas ? sms : kMaxCtas;
    cell->store(ctas);
  }
  const int rc = launch_pdl(kern, dim3(ctas), kDecodeThreads, S::kSmemBytes, a.stream,
                            static_cast<const uint8_t*>(a.c), static_cast<const uint8_t*>(a.kr),
                            static_cast<const __nv_bfloat16*>(a.q_c),
                            static_cast<const __nv_bfloat16*>(a.q_r),
                            static_cast<const __nv_bfloat16*>(a.q_sink), k);
  return rc != MLA_OK ? rc : launch_paged_join(k, ctas, 1, a);
}

// Clusters of `team` CTAs with one on an SM that are resident at a time; 0 if there are none or
// the runtime does not say, which is no error of the call. Asked until known for each size.
template <int DC, int DR>
int team_slots(int team) {
  using S = DecodeShape<DC, DR, true, true>;
  static_assert(S::kSmemBytes > 232448 / 2, "one CTA per SM");
  static PerDevice known[9];
  std::atomic<int>* cell = known[team].cell();
  if (!cell) return 0;
  int n = cell->load();
  if (n == 0) {
    auto kern = paged_decode_kernel<DC, DR, true, true>;
    cudaError_t e =
        cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, S::kSmemBytes);
    if (e == cudaSuccess) {
      cudaLaunchConfig_t cfg = {};
      cfg.gridDim = dim3(kMaxCtas / team * team);
      cfg.blockDim = dim3(kDecodeThreads);
      cfg.dynamicSmemBytes = S::kSmemBytes;
      cudaLaunchAttribute attr[1];
      attr[0].id = cudaLaunchAttributeClusterDimension;
      attr[0].val.clusterDim.x = team;
      attr[0].val.clusterDim.y = 1;
      attr[0].val.clusterDim.z = 1;
      cfg.attrs = attr;
      cfg.numAttrs = 1;
      e = cudaOccupancyMaxActiveClusters(&n, kern, &cfg);
    }
    if (e != cudaSuccess) {
      (void)cudaGetLastError();  // the call goes on without teams of this size
      return 0;
    }
    n = n < kMaxCtas / team ? n : kMaxCtas / team;
    cell->store(n);
  }
  return n;
}

// The same in teams of `team` CTAs (a cluster: 1, 2, 4 or 8), up to `teams` of them.
template <int DC, int DR>
int launch_teams(const PagedAttnArgs& a, int team, int teams) {
  using S = DecodeShape<DC, DR, true, true>;
  const PagedP<true> k = paged_params<true>(a, kBN, DC);
  auto kern = paged_decode_kernel<DC, DR, true, true>;
  static PerDevice known;  // the kernel's shared memory, set once
  std::atomic<int>* cell = known.cell();
  if (!cell) return MLA_ERR_CUDA;
  cudaError_t e = cudaSuccess;
  if (cell->load() == 0) {
    e = cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, S::kSmemBytes);
    if (e == cudaSuccess) cell->store(1);
  }
  if (e == cudaSuccess) {
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3(team * teams);
    cfg.blockDim = dim3(kDecodeThreads);
    cfg.dynamicSmemBytes = S::kSmemBytes;
    cfg.stream = a.stream;
    cudaLaunchAttribute attr[2];
    attr[0].id = cudaLaunchAttributeClusterDimension;
    attr[0].val.clusterDim.x = team;
    attr[0].val.clusterDim.y = 1;
    attr[0].val.clusterDim.z = 1;
    attr[1].id = cudaLaunchAttributeProgrammaticStreamSerialization;  // see grid_dep_sync
    attr[1].val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = attr;
    cfg.numAttrs = 2;
    e = cudaLaunchKernelEx(&cfg, kern, static_cast<const uint8_t*>(a.c),
                           static_cast<const uint8_t*>(a.kr),
                           static_cast<const __nv_bfloat16*>(a.q_c),
                           static_cast<const __nv_bfloat16*>(a.q_r),
                           static_cast<const __nv_bfloat16*>(a.q_sink), k);
  }
  if (e != cudaSuccess) {
    (void)cudaGetLastError();
    set_last_cuda_error(e);
    return MLA_ERR_CUDA;
  }
  return MLA_OK;
}

template <int DR>
int pick_teams(const PagedAttnArgs& a, int team, int teams) {
  switch (a.d_c) {
    case 64: return launch_teams<64, DR>(a, team, teams);
    case 128: return launch_teams<128, DR>(a, team, teams);
    case 192: return launch_teams<192, DR>(a, team, teams);
    case 256: return launch_teams<256, DR>(a, team, teams);
    default: return MLA_ERR_UNSUPPORTED;
  }
}

template <int DR, bool WIN>
int pick_decode(const PagedAttnArgs& a) {
  switch (a.d_c) {
    case 64: return launch_decode<64, DR, WIN>(a);
    case 128: return launch_decode<128, DR, WIN>(a);
    case 192: return launch_decode<192, DR, WIN>(a);
    case 256: return launch_decode<256, DR, WIN>(a);
    default: return MLA_ERR_UNSUPPORTED;
  }
}

}  // namespace
}  // namespace vmla
