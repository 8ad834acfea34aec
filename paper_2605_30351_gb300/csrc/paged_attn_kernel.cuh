// Attention of ragged streams' newest tokens over a paged latent cache, on the
// sm_103a tensor cores (Eq. score; App. E).
//
// Every (token, head) row of a stream scores the same latents, so a stream's
// rows stack along M and a key tile is read once per 128 of them:
//     S = [q_c | q_r] . [c | k]^T      K = d_c + d_r
//     P = exp2(S * log2(e)/sqrt(d_h) - m)   running maximum and sum in fp32, the sum
//                                      over unrounded weights; P is rounded to
//                                      bf16 (the type of c, as the MMA takes both
//                                      operands of one type). That rounding is as large
//                                      as the output's and independent of it: the
//                                      results' errors are up to sqrt(2) times those of
//                                      fp32 weights, where many keys weigh alike
//                                      (measured 1.0 - 1.25; simulated 1.09 - 1.42)
//     O += P . c                       N = d_c, c read again from the same tile
//
// Work is split evenly whatever the streams look like: all (row tile, key block)
// pairs of the call form one sequence, and each CTA (or pair of CTAs) takes a
// share of consecutive pairs of equal cost. A chunk of thousands of tokens, one
// token of one long stream and hundreds of ragged streams run on the same grid of
// one CTA per SM. A row tile that lies in one share is finished there; one that several
// shares cut writes unnormalised fp32 partial rows with their maximum and sum to
// the workspace, and paged_join_kernel adds them up in order. The shares depend
// on q_start and lens only, which every CTA reads for itself: no plan kernel, no
// host round trip, and the same result from call to call.
//
//   warp 0     finds the pages of a key block and copies them by TMA into a ring
//              of stages (one box per page and 64 columns). A row tile's Q takes
//              its turn in the same ring, so it is on its way while the previous
//              tile's last blocks are computed
//   warp 1     clears rows of a stage that hold no token of the stream (they may
//              hold NaN, and 0 * NaN would reach O), issues the score MMAs
//   warp 2     issues O += P V; of pairs with a window it does the clearing
//   warps 4-7  move Q from the ring to its place, then the softmax: thread i owns
//              row i. It copies a block's scores to registers at once, so the next
//              block's are computed while it works on the exponentials. Two threads
//              per row, and two groups of warps that take blocks in turns, were
//              both slower (a 4,680-token chunk on 32,760 keys at d_c = 192: 936
//              and 840 us against 809): what they save in a block's latency they
//              lose to exchanging maxima, registers and power.
// Pairs (CL = 2): two consecutive row tiles walk the same key blocks; each CTA
// fetches half of the boxes and multicasts them to both. At d_c = 512 the two
// CTAs of a pair share one row tile instead: each fetches 256 columns of c (the first
// k too), holds Q's and O's columns that go with them, and sends the other its part
// of the scores, which both add up (fp32; the same sum in both). 5 drafted tokens of
// 16 streams took 44.4 us with all scores computed in both CTAs, 33.5 us so.
//
// Pages that do not divide a block (24, 48 or 100 tokens) take one block each, copied as a
// box of BN rows: 2 x 500 tokens on 8,000 keys 316, 151 and 80 us, with pages of 16, 32, 64
// or 128 tokens 59 - 61 us.
//
// Measured on the GPU (12 heads, d_c = 192, d_r = 32): a chunk of 4,680 tokens on 32,760 keys
// 765 - 834 us in short runs (1.53 TFLOP: 1,835 - 2,000 TFLOP/s, 0.97 - 1.06 of the
// measured cuBLAS burst rate) and 850 us in long ones, which hold the GPU at its
// power limit; bound by the tensor pipe; at d_c = 256 and 512 1,415 and 4,786 us. 9 ragged
// prompts of up to 333 tokens on up to 5,001 keys (16 heads, d_c = 128, d_r = 64) 48 - 54
// us: 27 blocks a CTA take about 31 of them, bound by the softmax's latency and the MMAs
// together (tensor pipe 47 % active), the rest is the start, the join and cut tiles. 5
// drafted tokens of 16 streams (16 heads, d_c = 512, d_r = 64) 33.4 us, on 32,000 keys each
// 77 us
// (3.5 TB/s): 1.2 us for a block of 64 keys in turn through score MMAs (64 keys a
// step run at half rate), the exchange and the softmax, and 15 us of start, first
// copies and join.
//
// With a sliding window (WIN; App. D.4) a row sees the sinks j < S and e - w <= j < e, e the
// end of its block of the mask. A tile's key blocks are then two runs, the sinks' pages and
// those from the first row's window on (tile_span), and the row masks cut both ends; hidden
// keys may be NaN, so their rows of c are cleared before the output MMAs. The sinks may have
// positional queries of their own (App. D.5: k is stored rotated at absolute times, and a
// second rotation of q_r puts the sinks next to the window): a q_r tile more, in TMEM where it
// fits, for the columns that hold sinks. What a tile costs stops growing where its window is
// full, so the shares' cost has a knee (Cost<true>).
// Measured on the GPU: 4 x 4,680 tokens, a sink frame of 1,560 and the newest 9,360 tokens (12
// heads, d_c = 192, d_r = 32; 2.04 TFLOP) 1.04 ms in short runs (1,960 TFLOP/s, 1.03 of the
// measured burst rate; tensor pipe 83 % active under ncu) and 1.14 - 1.18 ms at the power limit;
// 9 prompts of up to 3,333 tokens, window 1,024, 4 sinks (16 heads, d_c = 128, d_r = 64) 164 -
// 180 us: 9 blocks of 2,100 - 2,500 clocks a tile, the softmax's (1,400 - 2,000 of them), and
// 6,500 between tiles (next segment, Q to TMEM, the last output); 28,000 tokens, window 4,096 (8
// heads, d_c = 256) 743 us: two stages of 73 KB do not hide the copies (as without a window);
// 5 drafted tokens of 16 streams, window 4,096 (16 heads, d_c = 512) 33.3 us.
// Not kept: blocks of 32 keys at a window's ends (205 -> 208 us for the prompts, chunks 1,135 ->
// 1,323); at d_c <= 128 Q in shared memory with the next tile's scores ahead of this one's
// output (2 % faster on average, 3 % slower where windows are long); Q copied to TMEM before
// the last block's weights (5 - 9 % slower with the votes that it needs).

#pragma once

#include <type_traits>

#include "internal.h"
#include "paged_attn.cuh"
#include "ptx_sm103.cuh"

namespace vmla {
namespace {

constexpr int kThreads = 256;  // 8 warps (the fourth: with a window a look at the metadata)
constexpr float kRescaleLog2 = 8.0f;

template <int DC, int DR, bool WIN>
struct PagedShape {
  // Keys per block: 64 only where 128 do not fit. A score MMA of 64 keys takes about
  // as long as one of 128 (71 clocks for each step of 16 values).
  static constexpr int BN = DC > 256 ? 64 : 128;
  static constexpr int DV = DC > 256 ? 256 : DC;   // output columns per CTA
  static constexpr int DK = DV + DR;               // c columns of its scores: the same
  static constexpr int kSplit = DC / DV;           // CTAs that share a row tile
  static constexpr int kTileBytes = BN * DK * 2;   // one stage
  static constexpr int kCBox = BN * 128;           // [BN rows x 64 columns] of c
  static constexpr int kKrOff = DV * BN * 2;       // the d_r columns of a stage
  static constexpr int kBoxes = DV / 64 + 1;       // boxes per page
  static constexpr int kQStages = kBM / BN;        // stages that Q takes
  // TMEM columns: S, P (bf16, two a column), O, and Q as far as it fits; the rest
  // of Q stays in shared memory. Where everything fits (d_c up to 128) S has two
  // buffers and P takes the place of the scores it came from, so that the next
  // block's scores are there before this one's weights are: with little MMA work a
  // block the softmax sets the pace. (d_c = 512 with q_r in shared memory would fit
  // too: 34.8 us for 33.5.)
  static constexpr int kBufs = 2 * BN + DV + DK / 2 <= 512 ? 2 : 1;
  static constexpr int kTmemS = 0;
  static constexpr int kTmemP = kBufs == 2 ? 0 : BN;
  static constexpr int kTmemO = kBufs == 2 ? 2 * BN : BN + BN / 2;
  static constexpr int kTmemQ = kTmemO + DV;
  static constexpr bool kQrTmem = kTmemQ + DK / 2 <= 512;
  static constexpr int kQcFit = (512 - kTmemQ) * 2 / 64 * 64;
  static constexpr int kQcTmem = kQcFit < DV ? kQcFit : DV;
  static constexpr int kQcSmem = DV - kQcTmem;
  static constexpr int kQKrOff = kQcSmem * kBM * 2;
  // the sinks' own q_r: behind Q in TMEM where it fits, else in shared memory
  static constexpr int kTmemQs = kTmemQ + DK / 2;
  static constexpr bool kQsTmem = kTmemQs + DR / 2 <= 512;
  static constexpr int kQsOff = kQrTmem ? 0 : kQKrOff + kBM * DR * 2;
  static constexpr int kQBytes = kQsOff + (WIN && !kQsTmem ? kBM * DR * 2 : 0);
  // a block's partial scores from the peer, fp32 as [64 / 4][128 rows][4 keys]; two of it
  static constexpr int kXBytes = kSplit > 1 ? BN * kBM * 4 : 0;
  static constexpr int kBarBytes = 512;  // barriers and small words
  static constexpr int kSmemCap = 232448;
  static constexpr int kFit =
      (kSmemCap - 1024 - kBarBytes - kQBytes - 2 * kXBytes) / kTileBytes;
  static constexpr int kMaxStages = BN == 128 ? 4 : 6;
  static constexpr int kStages = kFit > kMaxStages ? kMaxStages : kFit;
  static constexpr int kSmemBytes =
      1024 + kQBytes + kTileBytes * kStages + 2 * kXBytes + kBarBytes;
  static constexpr uint32_t kTmemCols = 512;
  static constexpr uint32_t kKrSw = DR == 32 ? kSw64 : kSw128;
  static constexpr uint32_t kKrRow = DR * 2;
  static constexpr uint32_t kKrSbo = 8 * kKrRow;
  static constexpr uint32_t kIdescQK = idesc_bf16_f32(kBM, BN, false, false);
  static constexpr uint32_t kIdescPV = idesc_bf16_f32(kBM, DV, false, true);
  static_assert(kTmemQ + kQcTmem / 2 <= 512 && kStages >= 2 && kStages >= kQStages,
                "TMEM and stages must fit");
  static_assert(!WIN || (kBM * DR * 2 <= kTileBytes && kStages > kQStages),
                "the sinks' q_r takes one stage, beside Q's");
  static_assert(kTileBytes % 1024 == 0 && kKrOff % 1024 == 0 && kQKrOff % 1024 == 0 &&
                    kQBytes % 1024 == 0,
                "swizzle-atom alignment");
};

// The map of the sinks' own q_r, where there may be one.
struct NoMap {};
template <bool WIN>
using SinkMap = std::conditional_t<WIN, CUtensorMap, NoMap>;

template <int DC, int DR, int CL, bool WIN, bool KEYS>
__global__ void __launch_bounds__(kThreads, 1)
    paged_attn_kernel(const __grid_constant__ CUtensorMap tm_c,
                      const __grid_constant__ CUtensorMap tm_kr,
                      const __grid_constant__ CUtensorMap tm_qc,
                      const __grid_constant__ CUtensorMap tm_qr,
                      const __grid_constant__ SinkMap<WIN> tm_qs, const PagedP<WIN> p) {
  using S = PagedShape<DC, DR, WIN>;
  constexpr int BN = S::BN, DV = S::DV, NST = S::kStages, QST = S::kQStages, NB = S::kBufs;
  constexpr int TR = kBM * CL / S::kSplit;  // rows of a CTA's, or a pair's, tile
  constexpr int MC = S::kSplit == 1 ? CL : 1;  // CTAs that share a stage's boxes
  // With a window the rows of c that a tile does not see are cleared between the weights and
  // the output, beside the next scores, where tiles are long (pairs: four chunks 1,100 -> 1,050
  // us, a prompt of 28,000 tokens 780 -> 760); else before the scores, by the warp that has the
  // code at hand (19 tokens of 3 streams 29.2 us, 30.0 so).
  constexpr bool kLate = WIN && CL == 2 && S::kSplit == 1;
  constexpr uint16_t kPair = static_cast<uint16_t>((1u << CL) - 1u);
  static_assert(S::kSplit == 1 || CL == S::kSplit, "split tiles take a pair");
  static_assert((2 * NST + 3 * NB + 12) * 8 + 64 + 2 * sizeof(Place<WIN>) + 8 <= S::kBarBytes,
                "barriers, the search's sums, the share's ends and two words fit");
  extern __shared__ uint8_t smem_raw[];
  uint8_t* smem = align_smem_1024(smem_raw);
  uint8_t* sQ = smem;
  uint8_t* sKV = smem + S::kQBytes;
  uint8_t* sX = sKV + NST * S::kTileBytes;
  uint64_t* bars = reinterpret_cast<uint64_t*>(sX + 2 * S::kXBytes);
  uint64_t* q_ready = bars;
  uint64_t* kv_full = bars + 1;
  uint64_t* kv_empty = kv_full + NST;
  uint64_t* s_free = kv_empty + NST;
  uint64_t* s_full = s_free + 1;           // [NB] each: by the buffer of the block,
  uint64_t* p_full = s_full + NB;          // so that a waiter one block behind still
  uint64_t* pv_done = p_full + NB;         // finds the phase it waits for
  uint64_t* mma_drain = pv_done + NB;      // [2]: one per issuing thread
  uint64_t* x_full = mma_drain + 2;        // [2][4]: a warp's scores from the peer
  long long* scratch = reinterpret_cast<long long*>(x_full + 8);  // [8]
  Place<WIN>* ends = reinterpret_cast<Place<WIN>*>(scratch + 8);               // [2]
  uint32_t* tmem_slot = reinterpret_cast<uint32_t*>(ends + 2);
  volatile int* abort_flag = reinterpret_cast<volatile int*>(tmem_slot + 1);

  const int warp = threadIdx.x >> 5;
  const int lane = threadIdx.x & 31;
  const WaitCtx wc{abort_flag, p.status};

  if (threadIdx.x == 0) {
    mbar_init(q_ready, kBM);
    for (int s = 0; s < NST; ++s) {
      mbar_init(&kv_full[s], 1);
      mbar_init(&kv_empty[s], MC);
    }
    mbar_init(s_free, kBM);
    for (int i = 0; i < NB; ++i) {
      mbar_init(&s_full[i], 1);
      mbar_init(&p_full[i], kBM);
      mbar_init(&pv_done[i], 1);
    }
    mbar_init(&mma_drain[0], 1);
    mbar_init(&mma_drain[1], 1);
    if (S::kSplit > 1)
      for (int i = 0; i < 8; ++i) mbar_init(&x_full[i], 1);
    *abort_flag = 0;
    fence_mbar_init();
    tma_prefetch_desc(&tm_c);
    tma_prefetch_desc(&tm_kr);
    tma_prefetch_desc(&tm_qc);
    tma_prefetch_desc(&tm_qr);
    if constexpr (WIN)
      if (p.turned) tma_prefetch_desc(&tm_qs);
  }
  if (warp == 1) {
    tmem_alloc(tmem_slot, S::kTmemCols);
    tmem_relinquish();
  }
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tmem = *tmem_slot;
  // the peer's barriers must be initialised before any multicast lands
  if constexpr (CL > 1) cluster_sync();
  grid_dep_sync();
  const int crank = CL > 1 ? static_cast<int>(cluster_ctarank()) : 0;
  const int first_row = S::kSplit == 1 ? crank * kBM : 0;  // of the pair's tile
  const int vpart = S::kSplit > 1 ? crank : 0;              // of c's columns
  const bool has_r = vpart == 0;  // the first of a split tile's CTAs adds q_r . k
  if (!WIN && blockIdx.x == 0) check_streams<WIN>(p, threadIdx.x, kThreads);
  if (threadIdx.x < 2) p.part_desc[2 * blockIdx.x + threadIdx.x] = make_int4(0, 0, 0, 0);
  const long long share =
      find_share<BN, TR, WIN>(p, blockIdx.x / CL, gridDim.x / CL, scratch, ends);
  Walk<BN, TR, WIN> walk(p, ends);
  Segment<WIN> g;
  bool ok = true;
  int it = 0;  // key blocks so far: the phases of the per-block barriers
  auto phase = [](int block) { return static_cast<uint32_t>(block / NB) & 1u; };
  int sc = 0;  // ring stages so far, Q's included: the phases of kv_full, kv_empty
  // a segment with blocks of the sinks has a stage more in front: their own q_r
  auto own_qr = [&](const Segment<WIN>& sg) {
    if constexpr (WIN) return p.turned && sg.kb0 < sg.at.sb ? 1 : 0;
    return 0;
  };

  if (warp < 4) {
    if (warp == 0) {
      // ------------------------------------------------------------ producer
      const int page_shift = 31 - __clz(p.page_tokens);  // pages that divide a block
      auto acquire = [&]() {  // stage sc is free
        bool free = true;
        if (sc >= NST) {
          if constexpr (MC == 1)
            free = mbar_wait(&kv_empty[sc % NST], ((sc / NST) - 1) & 1, wc);
          else  // the peer's threads arrive on it too
            free = mbar_wait_cluster(&kv_empty[sc % NST], ((sc / NST) - 1) & 1, wc);
        }
        return __all_sync(0xffffffffu, free);
      };
      while (ok && walk.next(g)) {
        const int rows = g.st.n * p.heads;
        // a lane per page of a block, looked up one block ahead of its copies
        const int* table = p.table + static_cast<size_t>(g.s) * p.max_pages;
        BlockPos<BN> pos(p, first_block(g));
        auto boxes_at = [&](const BlockPos<BN>& at) {  // pages of a block that hold tokens
          const int valid = min(at.rows(p), held_to(p, g, at.token(p)) - at.token(p));
          return p.per_group == 1 ? (valid > 0 ? 1 : 0)
                                  : (max(valid, 0) + p.page_tokens - 1) >> page_shift;
        };
        auto look_up = [&](const BlockPos<BN>& at) {
          return lane < boxes_at(at) ? table[page_index(p, g.at, at.grp * p.per_group + lane)] : -1;
        };
        int page_ahead = look_up(pos);
        for (int q = 0; q < QST; ++q, ++sc) {
          ok = acquire();
          if (!ok) break;
          const int r0 = g.tile * TR + first_row + q * BN;
          const int boxes = max(0, min(BN / 32, (rows - r0 + 31) / 32));
          uint8_t* st = sKV + (sc % NST) * S::kTileBytes;
          uint64_t* full = &kv_full[sc % NST];
          if (lane == 0) {
            if (boxes)
              mbar_arrive_expect_tx(full, boxes * 32 * (has_r ? S::DK : DV) * 2);
            else
              mbar_arrive(full);
          }
          __syncwarp();
          for (int bx = lane; bx < boxes * S::kBoxes; bx += 32) {
            const int i = bx / S::kBoxes, cb = bx - i * S::kBoxes;
            const int r = g.st.q0 * p.heads + r0 + 32 * i;
            if (cb < DV / 64)
              tma_load_2d(st + cb * S::kCBox + i * 32 * 128, &tm_qc, full, vpart * DV + cb * 64,
                          r);
            else if (has_r)
              tma_load_2d(st + S::kKrOff + i * 32 * S::kKrRow, &tm_qr, full, 0, r);
          }
        }
        if constexpr (WIN) {
          if (ok && own_qr(g)) {
            ok = acquire();
            if (ok) {
              const int r0 = g.tile * TR + first_row;
              const int boxes = has_r ? max(0, min(kBM / 32, (rows - r0 + 31) / 32)) : 0;
              uint64_t* full = &kv_full[sc % NST];
              if (lane == 0) {
                if (boxes)
                  mbar_arrive_expect_tx(full, boxes * 32 * DR * 2);
                else
                  mbar_arrive(full);
              }
              __syncwarp();
              if (lane < boxes)
                tma_load_2d(sKV + (sc % NST) * S::kTileBytes + lane * 32 * S::kKrRow, &tm_qs, full, 0,
                            g.st.q0 * p.heads + r0 + 32 * lane);
              ++sc;
            }
          }
        }
        if (!ok) break;
        for (int kb = g.kb0; kb < g.kb1; ++kb, ++sc) {
          const int boxes = boxes_at(pos), sub = pos.sub, page_now = page_ahead;
          next_block<BN>(p, g, kb, pos);
          if (kb + 1 < g.kb1) page_ahead = look_up(pos);
          ok = acquire();
          if (!ok) break;
          uint8_t* kv = sKV + (sc % NST) * S::kTileBytes;
          uint64_t* full = &kv_full[sc % NST];
          if (lane == 0) {
            if (boxes)
              mbar_arrive_expect_tx(full, boxes * p.box_rows * (has_r ? S::DK : DV) * 2);
            else
              mbar_arrive(full);
          }
          __syncwarp();
          for (int b0 = 0; b0 < boxes * S::kBoxes; b0 += 32) {
            const int bx = b0 + lane, i = bx / S::kBoxes, cb = bx - i * S::kBoxes;
            const int page = __shfl_sync(0xffffffffu, page_now, i & 31);
            if (i >= boxes || (MC > 1 && (bx & 1) != crank)) continue;
            int r = p.pages * p.page_tokens;  // past the pool: zeros
            if (page >= 0 && page < p.pages)
              r = page * p.page_tokens + sub * BN;
            else
              record_status(p.status, MLA_ERR_RANGE);
            const bool is_c = cb < DV / 64;
            if (!is_c && !has_r) continue;
            uint8_t* dst = is_c ? kv + cb * S::kCBox + i * p.box_rows * 128
                                : kv + S::kKrOff + i * p.box_rows * static_cast<int>(S::kKrRow);
            const CUtensorMap* map = is_c ? &tm_c : &tm_kr;
            const int x = is_c ? vpart * DV + cb * 64 : 0;
            if constexpr (MC == 1)
              tma_load_2d(dst, map, full, x, r);
            else
              tma_load_2d_mc(dst, map, full, x, r, kPair);
          }
        }
      }
      // every stage's last use must be released before the CTA may exit
      for (int st = 0; st < NST && st < sc && !*abort_flag; ++st)
        mbar_wait(&kv_empty[st], (((sc - st + NST - 1) / NST) - 1) & 1, wc);
      if (*abort_flag)  // let every copy this CTA started land before exit
        for (int u = sc > NST ? sc - NST : 0; u < sc; ++u)
          mbar_wait_drain(&kv_full[u % NST], (u / NST) & 1, p.status);
      __syncwarp();
    } else if (warp == 1) {
      // ---------------------------------------------------------- QK issuer
      const uint32_t qa = smem_u32(sQ);
      int seg = 0;
      while (ok && walk.next(g)) {
        ok = __all_sync(0xffffffffu, mbar_wait(q_ready, seg & 1, wc));
        ++seg;
        if (!ok) break;
        // Q has left its stages: give them back, to both CTAs of a pair
        for (int q = 0; q < QST + own_qr(g); ++q, ++sc)
          if (lane < MC) {
            if constexpr (MC == 1)
              mbar_arrive(&kv_empty[sc % NST]);
            else
              mbar_arrive_cluster(dsmem_addr(smem_u32(&kv_empty[sc % NST]), lane));
          }
        BlockPos<BN> pos(p, first_block(g));
        // where the keys end that the tile's first and last row see; its first behind the sinks
        int first_end = 0, last_end = 0, tile_low = 0;
        if constexpr (WIN && !kLate) {
          const int a = g.st.len - g.st.n;
          first_end = keys_seen<WIN>(p, a + p.by_heads(g.tile * TR), g.st);
          last_end = keys_seen<WIN>(
              p, a + p.by_heads(min(g.st.n * p.heads, (g.tile + 1) * TR) - 1), g.st);
          tile_low = first_key(p, first_end, g.st.gone);
        }
        for (int kb = g.kb0; kb < g.kb1; ++kb, ++it, ++sc, next_block<BN>(p, g, kb - 1, pos)) {
          const int st = sc % NST;
          uint8_t* kv = sKV + st * S::kTileBytes;
          const int token = pos.token(p);
          const int valid = max(0, min(pos.rows(p), held_to(p, g, token) - token));
          ok = __all_sync(0xffffffffu, mbar_wait(&kv_full[st], (sc / NST) & 1, wc));
          if (!ok) break;
          if constexpr (WIN && !kLate) {
            const uint4 zero = make_uint4(0u, 0u, 0u, 0u);
            // nothing to clear in most blocks: all rows hold tokens that some row sees
            if (valid < BN || tile_hides_some<BN>(p, g, kb, token, tile_low, last_end)) {
#pragma unroll 1
              for (int q = 0; q < BN / 32; ++q) {
                const int i = q * 32 + lane;
                const unsigned hid = __ballot_sync(
                    0xffffffffu,
                    i >= valid || tile_hides(p, g, kb, token + i, first_end, last_end));
                if (hid)
                  for (int cb = 0; cb < DV / 64; ++cb)
                    for (int j = lane; j < 32 * 8; j += 32)
                      if (hid >> (j >> 3) & 1)
                        *reinterpret_cast<uint4*>(kv + cb * S::kCBox + q * 32 * 128 + j * 16) =
                            zero;
              }
              fence_proxy_async_smem();
              __syncwarp();
            }
          } else if (!WIN && valid < BN) {
            const uint4 zero = make_uint4(0u, 0u, 0u, 0u);
            for (int cb = 0; cb < DV / 64; ++cb)
              for (int i = valid * 8 + lane; i < BN * 8; i += 32)
                *reinterpret_cast<uint4*>(kv + cb * S::kCBox + i * 16) = zero;
            fence_proxy_async_smem();
            __syncwarp();
          }
          // S's previous contents have been read: the scores by the softmax, or with
          // two buffers the weights that took their place by their PV
          if (it >= NB)
            ok = __all_sync(0xffffffffu,
                            NB == 1 ? mbar_wait(s_free, (it - 1) & 1, wc)
                                    : mbar_wait(&pv_done[it % NB], phase(it - NB), wc));
          if (!ok) break;
          if (lane == 0) {
            tc_fence_after();
            const uint32_t ka = smem_u32(kv);
            const uint32_t d = tmem + S::kTmemS + (it % NB) * BN;
#pragma unroll
            for (int cb = 0; cb < DV / 64; ++cb)
#pragma unroll
              for (int k = 0; k < 4; ++k) {
                const uint64_t bd = sdesc(ka + cb * S::kCBox + k * 32, 16, 1024, kSw128);
                const uint32_t acc = (cb | k) != 0 ? 1u : 0u;
                if (cb < S::kQcTmem / 64)
                  umma_ts(d, tmem + S::kTmemQ + (cb * 4 + k) * 8, bd, S::kIdescQK, acc);
                else
                  umma_ss(d, sdesc(qa + (cb - S::kQcTmem / 64) * 16384 + k * 32, 16, 1024, kSw128),
                          bd, S::kIdescQK, acc);
              }
            // q_r . k of all columns; where sinks are among them, of the sinks' pages (the
            // first columns) with their own q_r
            int own = 0;
            if constexpr (WIN)
              if (p.turned && kb < g.at.sb) own = p.compact ? min(BN, g.at.cut - token) : BN;
            if (own == 0) {
#pragma unroll
              for (int k = 0; k < (has_r ? DR / 16 : 0); ++k) {
                const uint64_t bd = sdesc(ka + S::kKrOff + k * 32, 16, S::kKrSbo, S::kKrSw);
                if constexpr (S::kQrTmem)
                  umma_ts(d, tmem + S::kTmemQ + DV / 2 + k * 8, bd, S::kIdescQK, 1u);
                else
                  umma_ss(d, sdesc(qa + S::kQKrOff + k * 32, 16, S::kKrSbo, S::kKrSw), bd,
                          S::kIdescQK, 1u);
              }
            } else if (has_r) {
              for (int c0 = 0; c0 < BN; c0 = own) {  // [0, own), then [own, BN)
                const bool sinks = c0 == 0;
                const int n = sinks ? own : BN - own;
                const uint32_t idesc = idesc_bf16_f32(kBM, 0, false, false) |
                                       (static_cast<uint32_t>(n >> 3) << 17);
#pragma unroll
                for (int k = 0; k < DR / 16; ++k) {
                  const uint64_t bd =
                      sdesc(ka + S::kKrOff + c0 * S::kKrRow + k * 32, 16, S::kKrSbo, S::kKrSw);
                  if (sinks ? S::kQsTmem : S::kQrTmem)
                    umma_ts(d + c0, tmem + (sinks ? S::kTmemQs : S::kTmemQ + DV / 2) + k * 8, bd,
                            idesc, 1u);
                  else
                    umma_ss(d + c0,
                            sdesc(qa + (sinks ? S::kQsOff : S::kQKrOff) + k * 32, 16, S::kKrSbo,
                                  S::kKrSw),
                            bd, idesc, 1u);
                }
                if (!sinks) break;
              }
            }
            umma_commit(&s_full[it % NB]);
          }
          __syncwarp();
        }
      }
      if (!ok && lane == 0) {  // wait for every MMA issued before TMEM is freed
        umma_commit(&mma_drain[0]);
        mbar_wait_drain(&mma_drain[0], 0, p.status);
      }
      __syncwarp();
    } else if (warp == 2) {
      // ---------------------------------------------------------- PV issuer
      if constexpr (kLate) {
        // Before an output the warp clears the rows of c that no row of the tile sees (there
        // are none in most blocks): what they score is masked, but they may hold NaN, and
        // 0 * NaN would reach O. It finds them while the weights are computed. (It cannot wait
        // for the copies alone: the stage's phase before may be a Q that it did not wait for.)
        while (ok && walk.next(g)) {
          sc += QST + own_qr(g);
          const int a = g.st.len - g.st.n;
          const int first_end = keys_seen<WIN>(p, a + p.by_heads(g.tile * TR), g.st);
          const int last_end = keys_seen<WIN>(
              p, a + p.by_heads(min(g.st.n * p.heads, (g.tile + 1) * TR) - 1), g.st);
          const int tile_low = first_key(p, first_end, g.st.gone);
          BlockPos<BN> pos(p, first_block(g));
          for (int kb = g.kb0; kb < g.kb1; ++kb, ++it, ++sc, next_block<BN>(p, g, kb - 1, pos)) {
            const int token = pos.token(p);
            const int valid = max(0, min(pos.rows(p), held_to(p, g, token) - token));
            const bool some =
                valid < BN || tile_hides_some<BN>(p, g, kb, token, tile_low, last_end);
            unsigned hid[BN / 32] = {};
            if (some)
#pragma unroll
              for (int q = 0; q < BN / 32; ++q) {
                const int i = q * 32 + lane;
                hid[q] = __ballot_sync(
                    0xffffffffu,
                    i >= valid || tile_hides(p, g, kb, token + i, first_end, last_end));
              }
            // the weights are there, so the block's copies and scores are done
            ok = __all_sync(0xffffffffu, mbar_wait(&p_full[it % NB], phase(it), wc));
            if (!ok) break;
            if (some) {
              uint8_t* kv = sKV + (sc % NST) * S::kTileBytes;
              const uint4 zero = make_uint4(0u, 0u, 0u, 0u);
#pragma unroll
              for (int q = 0; q < BN / 32; ++q)
                if (hid[q])
                  for (int cb = 0; cb < DV / 64; ++cb)
                    for (int j = lane; j < 32 * 8; j += 32)
                      if (hid[q] >> (j >> 3) & 1)
                        *reinterpret_cast<uint4*>(kv + cb * S::kCBox + q * 32 * 128 + j * 16) =
                            zero;
              fence_proxy_async_smem();
              __syncwarp();
            }
            if (lane == 0) {
              tc_fence_after();
              const int st = sc % NST;
              const uint32_t va = smem_u32(sKV) + st * S::kTileBytes;
#pragma unroll
              for (int s = 0; s < BN / 16; ++s)
                umma_ts(tmem + S::kTmemO, tmem + S::kTmemP + (it % NB) * BN + s * 8,
                        sdesc(va + s * 2048, S::kCBox, 1024, kSw128), S::kIdescPV,
                        (kb > g.kb0 || s > 0) ? 1u : 0u);
              umma_commit_mc(&kv_empty[st], kPair);
              umma_commit(&pv_done[it % NB]);
            }
            __syncwarp();
          }
        }
        if (!ok && lane == 0) {
          umma_commit(&mma_drain[1]);
          mbar_wait_drain(&mma_drain[1], 0, p.status);
        }
      } else if (lane == 0) {
        while (ok && walk.next(g)) {
          sc += QST + own_qr(g);
          for (int kb = g.kb0; kb < g.kb1; ++kb, ++it, ++sc) {
            ok = mbar_wait(&p_full[it % NB], phase(it), wc);
            if (!ok) break;
            tc_fence_after();
            const int st = sc % NST;
            const uint32_t va = smem_u32(sKV) + st * S::kTileBytes;
#pragma unroll
            for (int s = 0; s < BN / 16; ++s)
              umma_ts(tmem + S::kTmemO, tmem + S::kTmemP + (it % NB) * BN + s * 8,
                      sdesc(va + s * 2048, S::kCBox, 1024, kSw128), S::kIdescPV,
                      (kb > g.kb0 || s > 0) ? 1u : 0u);
            if constexpr (MC == 1)
              umma_commit(&kv_empty[st]);
            else
              umma_commit_mc(&kv_empty[st], kPair);
            umma_commit(&pv_done[it % NB]);
          }
        }
        if (!ok) {
          umma_commit(&mma_drain[1]);
          mbar_wait_drain(&mma_drain[1], 0, p.status);
        }
      }
      __syncwarp();
    } else if (WIN && blockIdx.x == 0) {  // the warp without a role
      check_streams<WIN>(p, lane, 32);
      __syncwarp();
    }
  } else {
    // --------------------------------------------------- softmax (warps 4..7)
    const int quarter = warp & 3;  // TMEM lane quarter this warp may access
    const int r = quarter * 32 + lane;
    const uint32_t t_lane = static_cast<uint32_t>(quarter * 32) << 16;
    int xc = 0;  // blocks exchanged with the peer
    struct Row {
      int tile0, lrow, keys;  // the CTA's first row, this thread's, where its keys end
      int low;                // the first of them behind the sinks
      size_t grow;            // its place in q and o
      bool ok, warp_ok;       // the row exists; one of the warp's does
    };
    // The thread's row of a segment, and its Q, from the ring stage into TMEM
    // (row-major, two values a column) and shared memory (the swizzle the MMA
    // descriptors name). The score MMAs that read the previous Q are done: their
    // scores were awaited.
    auto load_row = [&](const Segment<WIN>& sg, Row& w) {
      const int rows = sg.st.n * p.heads;
      w.tile0 = sg.tile * TR + first_row;
      w.lrow = w.tile0 + r;
      w.ok = w.lrow < rows;
      w.warp_ok = __any_sync(0xffffffffu, w.ok);
      w.grow = static_cast<size_t>(sg.st.q0) * p.heads + (w.ok ? w.lrow : 0);
      w.keys = w.ok ? keys_seen<WIN>(p, sg.st.len - sg.st.n + p.by_heads(w.lrow), sg.st) : 0;
      if constexpr (WIN) w.low = first_key(p, w.keys, sg.st.gone);
      const int slot = sc + (QST > 1 ? r / BN : 0), rr = QST > 1 ? r % BN : r;
      if (!mbar_wait(&kv_full[slot % NST], (slot / NST) & 1, wc)) return false;
      if (w.warp_ok) {
        const uint8_t* st = sKV + (slot % NST) * S::kTileBytes;
        auto c_piece = [&](int i) {  // 16-byte piece i of the row's q_c
          return *reinterpret_cast<const uint4*>(st + (i / 8) * S::kCBox + rr * 128 +
                                                 (((i % 8) ^ (rr & 7)) * 16));
        };
        auto r_piece = [&](int i) {
          const int at = DR == 32 ? (i ^ ((rr >> 1) & 3)) : (i ^ (rr & 7));
          return *reinterpret_cast<const uint4*>(st + S::kKrOff + rr * S::kKrRow + at * 16);
        };
        constexpr int kTm = S::kQcTmem / 8, kRr = DR / 8;
        constexpr int kGrp = S::kQcTmem / 32 + (S::kQrTmem ? DR / 32 : 0);
#pragma unroll
        for (int gi = 0; gi < kGrp; ++gi) {
          uint4 v[4];
#pragma unroll
          for (int i = 0; i < 4; ++i)
            v[i] = gi < S::kQcTmem / 32 ? c_piece(4 * gi + i) : r_piece(4 * gi - kTm + i);
          tmem_st16(tmem + t_lane + S::kTmemQ + gi * 16, reinterpret_cast<const uint32_t*>(v));
        }
        if constexpr (!S::kQrTmem) {
#pragma unroll
          for (int c = 0; c < S::kQcSmem / 64; ++c)
#pragma unroll
            for (int i = 0; i < 8; ++i)
              *reinterpret_cast<uint4*>(sQ + c * 16384 + r * 128 + ((i ^ (r & 7)) * 16)) =
                  c_piece(kTm + c * 8 + i);
          uint8_t* dst = sQ + S::kQKrOff + r * S::kKrRow;
#pragma unroll
          for (int i = 0; i < kRr; ++i) {
            const int at = DR == 32 ? (i ^ ((r >> 1) & 3)) : (i ^ (r & 7));
            *reinterpret_cast<uint4*>(dst + at * 16) = r_piece(i);
          }
          fence_proxy_async_smem();
        }
        if constexpr (S::kQcTmem > 0) tmem_wait_st();
      }
      if (own_qr(sg)) {
        const int at = (sc + QST) % NST;
        if (!mbar_wait(&kv_full[at], ((sc + QST) / NST) & 1, wc)) return false;
        if (w.warp_ok && has_r) {
          const uint8_t* st = sKV + at * S::kTileBytes;
          auto piece = [&](int i) {
            return *reinterpret_cast<const uint4*>(
                st + r * S::kKrRow + (DR == 32 ? (i ^ ((r >> 1) & 3)) : (i ^ (r & 7))) * 16);
          };
          if constexpr (S::kQsTmem) {
#pragma unroll
            for (int gi = 0; gi < DR / 32; ++gi) {
              uint4 v[4];
#pragma unroll
              for (int i = 0; i < 4; ++i) v[i] = piece(4 * gi + i);
              tmem_st16(tmem + t_lane + S::kTmemQs + gi * 16, reinterpret_cast<const uint32_t*>(v));
            }
            tmem_wait_st();
          } else {  // the stage's swizzle is the operand's
            uint8_t* dst = sQ + S::kQsOff + r * S::kKrRow;
#pragma unroll
            for (int i = 0; i < DR / 8; ++i)
              *reinterpret_cast<uint4*>(dst + i * 16) =
                  *reinterpret_cast<const uint4*>(st + r * S::kKrRow + i * 16);
            fence_proxy_async_smem();
          }
        }
      }
      tc_fence_before();
      mbar_arrive(q_ready);
      sc += QST + own_qr(sg);
      return true;
    };
    bool have = walk.next(g);
    if (!have && r == 0) p.part_desc[2 * blockIdx.x] = make_int4(0, 0, kPartEmpty, 0);
    Row w{};
    if (have) ok = load_row(g, w);
    while (ok && have) {
      float m_run = -INFINITY, l_run = 0.f;
      BlockPos<BN> pos(p, first_block(g));
      for (int kb = g.kb0; kb < g.kb1; ++kb, ++it, next_block<BN>(p, g, kb - 1, pos)) {
        View v{0, 0, 0};
        if constexpr (WIN) v = view_of(p, g, kb, pos.token(p), w.keys, w.low);
        if (!mbar_wait(&s_full[it % NB], phase(it), wc)) {
          ok = false;
          break;
        }
        tc_fence_after();
        if (!w.warp_ok) {  // none of the warp's rows exists: keep the barriers going
          if constexpr (NB == 1) {
            mbar_arrive(s_free);
            if (kb > g.kb0 && !mbar_wait(pv_done, (it - 1) & 1, wc)) {
              ok = false;
              break;
            }
          }
          mbar_arrive(&p_full[it % NB]);
          continue;
        }
        uint32_t sr[BN];
#pragma unroll
        for (int c = 0; c < BN / 32; ++c)
          tmem_ld32(tmem + t_lane + S::kTmemS + (it % NB) * BN + c * 32,
                    *reinterpret_cast<uint32_t(*)[32]>(&sr[c * 32]));
        tmem_wait_ld();
        if constexpr (NB == 1) {
          tc_fence_before();
          mbar_arrive(s_free);  // the next block's scores may land
        }
        float sv[BN];
#pragma unroll
        for (int c = 0; c < BN; ++c) sv[c] = __uint_as_float(sr[c]);
        if constexpr (S::kSplit > 1) {
          // The scores over all of c are this CTA's and the peer's: each sends its own
          // (row by row, warp by warp) and adds what it gets. A buffer is written again
          // two blocks later: by then the peer's scores of the block between are here,
          // and it sent them after it had read these. Plain stores with a released
          // arrival took 0.5 us a block more; sending a block ahead of its softmax,
          // which spills registers, 0.15 us.
          const uint32_t off = (xc & 1) * S::kXBytes + r * 16;
          const uint32_t to = dsmem_addr(smem_u32(sX) + off, crank ^ 1);
          uint64_t* full = &x_full[(xc & 1) * 4 + quarter];
          const uint32_t bar = dsmem_addr(smem_u32(full), crank ^ 1);
#pragma unroll
          for (int c = 0; c < BN / 4; ++c)
            st_async_v4(to + c * kBM * 16, bar, sv[4 * c], sv[4 * c + 1], sv[4 * c + 2],
                        sv[4 * c + 3]);
          if (lane == 0) mbar_arrive_expect_tx(full, 32 * BN * 4);
          if (!mbar_wait_cluster(full, (xc >> 1) & 1, wc)) {
            ok = false;
            break;
          }
          ++xc;
#pragma unroll
          for (int c = 0; c < BN / 4; ++c) {
            const float4 v = *reinterpret_cast<const float4*>(sX + off + c * kBM * 16);
            sv[4 * c] += v.x;
            sv[4 * c + 1] += v.y;
            sv[4 * c + 2] += v.z;
            sv[4 * c + 3] += v.w;
          }
        }
        int valid = min(pos.rows(p), w.keys - pos.token(p));
        bool sees = true;  // WIN: the row sees one of the block's keys
        if constexpr (WIN) {
          valid = min(pos.rows(p), v.valid);
          sees = v.sinks > 0 || max(v.low, 0) < valid;
          // Most blocks hide no keys, those at a window's ends a run or two: 32 keys at a time by a
          // bit each, or (KEYS, see keyed) key by key.
          if constexpr (KEYS) {
            if (v.low > 0 && v.sinks < BN) {
#pragma unroll
              for (int c = 0; c < BN; ++c)
                if (c < v.low && c >= v.sinks) sv[c] = -INFINITY;
            }
            if (valid < BN) {
#pragma unroll
              for (int c = 0; c < BN; ++c)
                if (c >= valid) sv[c] = -INFINITY;
            }
          } else if (v.low > 0 || valid < BN) {
#pragma unroll
            for (int q = 0; q < BN / 32; ++q) {
              const unsigned shown = low_bits(valid - 32 * q) &
                                     (~low_bits(v.low - 32 * q) | low_bits(v.sinks - 32 * q));
#pragma unroll
              for (int i = 0; i < 32; ++i)
                if (!(shown >> i & 1)) sv[32 * q + i] = -INFINITY;
            }
          }
        } else if (valid < BN) {
#pragma unroll
          for (int c = 0; c < BN; ++c)
            if (c >= valid) sv[c] = -INFINITY;
        }
        float m8[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) m8[i] = sv[i];
#pragma unroll
        for (int c = 8; c + 16 <= BN; c += 16)
#pragma unroll
          for (int i = 0; i < 8; ++i) m8[i] = fmax3(m8[i], sv[c + i], sv[c + 8 + i]);
#pragma unroll
        for (int i = 0; i < 8; ++i) m8[i] = fmaxf(m8[i], sv[BN - 8 + i]);
        const float mx = fmaxf(fmaxf(fmaxf(m8[0], m8[1]), fmaxf(m8[2], m8[3])),
                               fmaxf(fmaxf(m8[4], m8[5]), fmaxf(m8[6], m8[7])));
        const float m_blk = mx * p.scale_log2;
        // The running maximum moves only when a block exceeds it by more than
        // 2^8 (weights up to 256 are harmless in bf16 and fp32). A row that sees
        // no key of the first block sees none of the segment (it sees a prefix) and
        // has none; its weights are exp2(-inf) = 0. With a window the maximum begins
        // with the first block of which the row sees a key: what was added to O and to
        // the sum before are zeros.
        float alpha = 1.f;
        bool need = false;
        if (WIN ? m_run == -INFINITY : kb == g.kb0) {
          m_run = (WIN ? sees : valid > 0) ? fmaxf(m_blk, kLowest) : -INFINITY;
        } else if (m_blk > m_run + kRescaleLog2) {
          need = true;
          alpha = ex2_approx(m_run - m_blk);
          m_run = m_blk;
        }
        debug_count_rescale(need && w.ok, p.status);
        l_run *= alpha;
        const float neg_m = m_run == -INFINITY ? 0.f : -m_run;
        const uint64_t scale2 = f32x2_pack(p.scale_log2, p.scale_log2);
        const uint64_t negm2 = f32x2_pack(neg_m, neg_m);
        uint64_t l4[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) l4[i] = 0ull;
        uint32_t pk[BN / 2];
#pragma unroll
        for (int i = 0; i < BN / 2; ++i) {
          float t0, t1;
          f32x2_unpack(f32x2_fma(f32x2_pack(sv[2 * i], sv[2 * i + 1]), scale2, negm2), t0, t1);
          const float p0 = ex2_approx(t0);
          const float p1 = ex2_approx(t1);
          l4[i & 3] = f32x2_add(l4[i & 3], f32x2_pack(p0, p1));
          pk[i] = pack_bf16x2(p0, p1);
        }
        float l8[8];
#pragma unroll
        for (int i = 0; i < 4; ++i) f32x2_unpack(l4[i], l8[2 * i], l8[2 * i + 1]);
        l_run += ((l8[0] + l8[1]) + (l8[2] + l8[3])) + ((l8[4] + l8[5]) + (l8[6] + l8[7]));
        // the previous PV has read P (one buffer) and finished with O
        const bool rescale = __any_sync(0xffffffffu, need);
        if (kb > g.kb0 && (NB == 1 || rescale)) {
          if (!mbar_wait(&pv_done[(it - 1) % NB], phase(it - 1), wc)) {
            ok = false;
            break;
          }
          tc_fence_after();
          if (rescale) {
#pragma unroll 1
            for (int c = 0; c < DV / 32; ++c) {
              uint32_t ov[32];
              tmem_ld32(tmem + t_lane + S::kTmemO + c * 32, ov);
              tmem_wait_ld();
#pragma unroll
              for (int i = 0; i < 32; ++i)
                ov[i] = __float_as_uint(__uint_as_float(ov[i]) * alpha);
              tmem_st32(tmem + t_lane + S::kTmemO + c * 32, ov);
            }
          }
        }
#pragma unroll
        for (int c = 0; c < BN / 64; ++c)
          tmem_st32(tmem + t_lane + S::kTmemP + (it % NB) * BN + c * 32,
                    *reinterpret_cast<uint32_t(*)[32]>(&pk[c * 32]));
        tmem_wait_st();
        tc_fence_before();
        mbar_arrive(&p_full[it % NB]);
      }

      if (!ok) break;
      sc += g.kb1 - g.kb0;
      // The next segment's Q first, so that its scores are computed while this
      // one's O is written.
      const Row d = w;
      const bool starts = g.kb0 == 0, stops = g.kb1 == g.at.all, whole = starts && stops;
      const int n_rows = max(0, min(kBM, g.st.n * p.heads - d.tile0));
      const int row0 = g.st.q0 * p.heads + d.tile0;
      const bool many = static_cast<long long>(g.at.all) * BN > kManyShares * share;
      const bool by_row = many || n_rows <= kFewRows;
      have = walk.next(g);
      if (have) ok = load_row(g, w);
      // O: finished rows as bf16, a cut tile's as fp32 partial rows, stored as
      // [4 columns][rows] so that a warp's stores are contiguous
      ok = ok && mbar_wait(&pv_done[(it - 1) % NB], phase(it - 1), wc);
      if (!ok) break;
      tc_fence_after();
      const int slot = 2 * blockIdx.x + (starts ? 1 : 0);
      if (d.warp_ok) {
        // a row that saw no key is 0; a NaN sum stays one
        const float f = l_run == 0.f ? 0.f : 1.f / l_run;
        float* part = p.part_o + static_cast<size_t>(slot) * DV * kBM;
        __nv_bfloat16* dst = p.o + d.grow * DC + vpart * DV;
#pragma unroll 1
        for (int c = 0; c < DV / 32; ++c) {
          uint32_t ov[32];
          tmem_ld32(tmem + t_lane + S::kTmemO + c * 32, ov);
          tmem_wait_ld();
          if (d.ok && whole) {
#pragma unroll
            for (int i = 0; i < 2; ++i) {
              uint32_t x[8];
#pragma unroll
              for (int k = 0; k < 8; ++k)
                x[k] = pack_bf16x2(__uint_as_float(ov[16 * i + 2 * k]) * f,
                                   __uint_as_float(ov[16 * i + 2 * k + 1]) * f);
              if constexpr (WIN && DC > 128)
                if (p.o_wide) {
                  st_global_32(dst + c * 32 + i * 16, x);
                  continue;
                }
              *reinterpret_cast<uint4*>(dst + c * 32 + i * 16) = make_uint4(x[0], x[1], x[2], x[3]);
              *reinterpret_cast<uint4*>(dst + c * 32 + i * 16 + 8) =
                  make_uint4(x[4], x[5], x[6], x[7]);
            }
          } else if (d.ok && by_row) {
#pragma unroll
            for (int i = 0; i < 4; ++i) st_global_32(part + r * DV + c * 32 + i * 8, ov + 8 * i);
          } else if (d.ok) {
#pragma unroll
            for (int i = 0; i < 8; ++i)
              reinterpret_cast<float4*>(part)[(c * 8 + i) * kBM + r] =
                  make_float4(__uint_as_float(ov[4 * i]), __uint_as_float(ov[4 * i + 1]),
                              __uint_as_float(ov[4 * i + 2]), __uint_as_float(ov[4 * i + 3]));
          }
          __syncwarp();  // the next TMEM load is the whole warp's
        }
        if (!whole && d.ok) p.part_ml[slot * kBM + r] = make_float2(m_run, l_run);
        tc_fence_before();  // O was read before the next segment's first PV
      }
      if (!whole && r == 0)
        p.part_desc[slot] =
            make_int4(row0, n_rows, kPartHeld | (stops ? kPartEnds : 0), many ? 2 : by_row);
    }
  }

  tc_fence_before();
  __syncthreads();
  if (warp == 1) {
    tc_fence_after();
    tmem_dealloc(tmem, S::kTmemCols);
  }
  // neither CTA leaves while the other may still write into its shared memory
  if constexpr (CL > 1) cluster_sync();
}

template <int DC, int DR, int CL, bool WIN, bool KEYS = false>
int launch_paged(const PagedAttnArgs& a) {
  using S = PagedShape<DC, DR, WIN>;
  const PagedP<WIN> k = paged_params<WIN>(a, S::BN, S::DV);
  CUtensorMap tm_c, tm_kr;
  const unsigned long long rows = static_cast<unsigned long long>(a.pages) * a.page_tokens;
  if (!encode_map_2d_bf16(&tm_c, a.c, DC, rows, DC * 2ull, 64, k.box_rows,
                          CU_TENSOR_MAP_SWIZZLE_128B) ||
      !encode_map_2d_bf16(&tm_kr, a.kr, DR, rows, DR * 2ull, DR, k.box_rows,
                          DR == 32 ? CU_TENSOR_MAP_SWIZZLE_64B : CU_TENSOR_MAP_SWIZZLE_128B))
    return MLA_ERR_CUDA;
  SinkMap<WIN> tm_qs{};
  CUtensorMap tm_qc, tm_qr;  // boxes of 32 rows: short tiles fetch what they have
  const unsigned long long q_rows = static_cast<unsigned long long>(a.total) * a.heads;
  if (!encode_map_2d_bf16(&tm_qc, a.q_c, DC, q_rows, DC * 2ull, 64, 32,
                          CU_TENSOR_MAP_SWIZZLE_128B) ||
      !encode_map_2d_bf16(&tm_qr, a.q_r, DR, q_rows, DR * 2ull, DR, 32,
                          DR == 32 ? CU_TENSOR_MAP_SWIZZLE_64B : CU_TENSOR_MAP_SWIZZLE_128B))
    return MLA_ERR_CUDA;
  if constexpr (WIN) {
    if (!k.turned)
      tm_qs = tm_qr;
    else if (!encode_map_2d_bf16(
                 &tm_qs, a.q_sink, DR, q_rows, DR * 2ull, DR, 32,
                 DR == 32 ? CU_TENSOR_MAP_SWIZZLE_64B : CU_TENSOR_MAP_SWIZZLE_128B))
      return MLA_ERR_CUDA;
  }
  auto kern = paged_attn_kernel<DC, DR, CL, WIN, KEYS>;
  // resident CTAs of this instance (one per SM, whole clusters), asked once
  static PerDevice known;
  std::atomic<int>* cell = known.cell();
  if (!cell) return MLA_ERR_CUDA;
  int resident = cell->load();
  if (resident == 0) {
    cudaError_t e =
        cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, S::kSmemBytes);
    int n = 0;
    if (e == cudaSuccess) {
      cudaLaunchConfig_t oc = {};
      oc.gridDim = dim3(kMaxCtas / CL * CL);
      oc.blockDim = dim3(kThreads);
      oc.dynamicSmemBytes = S::kSmemBytes;
      cudaLaunchAttribute at[1];
      at[0].id = cudaLaunchAttributeClusterDimension;
      at[0].val.clusterDim.x = CL;
      at[0].val.clusterDim.y = 1;
      at[0].val.clusterDim.z = 1;
      oc.attrs = at;
      oc.numAttrs = 1;
      e = cudaOccupancyMaxActiveClusters(&n, kern, &oc);
    }
    if (e == cudaSuccess && n < 1) e = cudaErrorLaunchOutOfResources;
    if (e != cudaSuccess) {
      (void)cudaGetLastError();
      set_last_cuda_error(e);
      return MLA_ERR_CUDA;
    }
    resident = n * CL < kMaxCtas ? n * CL : kMaxCtas / CL * CL;
    cell->store(resident);
  }
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3(resident);
  cfg.blockDim = dim3(kThreads);
  cfg.dynamicSmemBytes = S::kSmemBytes;
  cfg.stream = a.stream;
  cudaLaunchAttribute attr[2];
  attr[0].id = cudaLaunchAttributeClusterDimension;
  attr[0].val.clusterDim.x = CL;
  attr[0].val.clusterDim.y = 1;
  attr[0].val.clusterDim.z = 1;
  attr[1].id = cudaLaunchAttributeProgrammaticStreamSerialization;  // see grid_dep_sync
  attr[1].val.programmaticStreamSerializationAllowed = 1;
  cfg.attrs = attr;
  cfg.numAttrs = 2;
  const cudaError_t e = cudaLaunchKernelEx(&cfg, kern, tm_c, tm_kr, tm_qc, tm_qr, tm_qs, k);
  if (e != cudaSuccess) {
    (void)cudaGetLastError();
    set_last_cuda_error(e);
    return MLA_ERR_CUDA;
  }
  return launch_paged_join(k, resident, CL, a);
}

// Two row tiles and more a slot of the pool on average: CTA pairs, which read each key
// tile from L2 once for 256 rows. Shorter ones would leave half a pair idle (ragged
// prompts 51 us with pairs, 60 without). Idle slots count as short streams here too: a
// 4,680-token chunk on 32,760 keys 820 us in a pool of 4 slots, 891 of 256.
inline bool takes_pairs(const PagedAttnArgs& a) {
  if (a.form != 0) return a.form == 2 * kBM;
  return static_cast<long long>(a.total) * a.heads >= 2ll * kBM * a.seqs;
}

// How a window's hidden keys leave a row's scores. Rows whose mask gives them a window each (token
// by token) take a bit a key; rows of a block of the mask agree on what they see, so a warp has
// one end of the window in a block at most and compares key by key. Pairs, windows of 500 / 2,000 /
// 8,000 / 30,000 keys, us by bits and by keys:
//   d_c     2 x 3,000 tokens, token by token                1 x 4,680 tokens, one block
//    64  50 / 82 / 215 / 703, 53 / 84 / 222 / 728      96 / 141 / 207 / 587,  88 / 134 / 206 / 600
//   128  57 / 101 / 272 / 887, 60 / 105 / 276 / 902   115 / 163 / 256 / 738, 102 / 152 / 255 / 741
//   192  63 / 106 / 275 / 889, 64 / 106 / 271 / 863   120 / 171 / 259 / 743, 115 / 166 / 249 / 726
//   256  83 / 164 / 478 / 1628, 84 / 166 / 489 / 1676 146 / 214 / 444 / 1340, 144 / 212 / 450 / 1375
// (128 with d_r = 64, the others with 32). Beyond d_c = 192 keys give no more than they cost (at
// 512 3 % less to 2 % more). Both in one kernel, by a branch, is 1 - 3 % slower token by token
// at 64 and 128.
inline bool keyed(const PagedAttnArgs& a) { return a.causal_block != 1; }

template <int DC, int DR, bool WIN>
int pick(const PagedAttnArgs& a) {
  if constexpr (PagedShape<DC, DR, WIN>::kSplit == 2) {
    return launch_paged<DC, DR, 2, WIN>(a);
  } else {
    if (!takes_pairs(a)) return launch_paged<DC, DR, 1, WIN>(a);
    if constexpr (WIN && DC <= 192)
      if (keyed(a)) return launch_paged<DC, DR, 2, WIN, true>(a);
    return launch_paged<DC, DR, 2, WIN>(a);
  }
}

template <int DR, bool WIN>
int pick_dc(const PagedAttnArgs& a) {
  switch (a.d_c) {
    case 64: return pick<64, DR, WIN>(a);
    case 128: return pick<128, DR, WIN>(a);
    case 192: return pick<192, DR, WIN>(a);
    case 256: return pick<256, DR, WIN>(a);
    case 512: return pick<512, DR, WIN>(a);
    default: return MLA_ERR_UNSUPPORTED;
  }
}

}  // namespace
}  // namespace vmla
