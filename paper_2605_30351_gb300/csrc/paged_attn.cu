// Attention of ragged streams' newest tokens over a paged latent cache, on the
// sm_103a tensor cores (Eq. score; App. E).
//
// Every (token, head) row of a stream scores the same latents, so a stream's
// rows stack along M and a key tile is read once per 128 of them:
//     S = [q_c | q_r] . [c | k]^T      K = d_c + d_r
//     P = exp2(S * log2(e)/sqrt(d_h) - m)   running maximum and sum in fp32, the sum
//                                      over unrounded weights; P is rounded to
//                                      bf16 (the type of c, as the MMA takes both
//                                      operands of one type): the results' errors are
//                                      1.0 to 1.3 times those of fp32 weights
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
//   warp 2     issues O += P V
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
#include <cmath>

#include "internal.h"
#include "paged_attn.cuh"
#include "ptx_sm103.cuh"

namespace vmla {
namespace {

constexpr int kThreads = 256;  // 8 warps (the fourth has no role)
constexpr float kRescaleLog2 = 8.0f;
constexpr int kJoinThreads = 512;
constexpr int kJoinGrid = kMaxCtas;
constexpr int kJoinCols = 16;  // columns of a warp's join item of 32 rows

template <int DC, int DR>
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
  static constexpr int kQBytes = kQrTmem ? 0 : kQKrOff + kBM * DR * 2;
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
  static_assert(kTileBytes % 1024 == 0 && kKrOff % 1024 == 0 && kQKrOff % 1024 == 0,
                "swizzle-atom alignment");
};

template <int DC, int DR, int CL>
__global__ void __launch_bounds__(kThreads, 1)
    paged_attn_kernel(const __grid_constant__ CUtensorMap tm_c,
                      const __grid_constant__ CUtensorMap tm_kr,
                      const __grid_constant__ CUtensorMap tm_qc,
                      const __grid_constant__ CUtensorMap tm_qr, const PagedK p) {
  using S = PagedShape<DC, DR>;
  constexpr int BN = S::BN, DV = S::DV, NST = S::kStages, QST = S::kQStages, NB = S::kBufs;
  constexpr int TR = kBM * CL / S::kSplit;  // rows of a CTA's, or a pair's, tile
  constexpr int MC = S::kSplit == 1 ? CL : 1;  // CTAs that share a stage's boxes
  constexpr uint16_t kPair = static_cast<uint16_t>((1u << CL) - 1u);
  static_assert(S::kSplit == 1 || CL == S::kSplit, "split tiles take a pair");
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
  Place* ends = reinterpret_cast<Place*>(scratch + 8);               // [2]
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
  if (blockIdx.x == 0) {
    check_q_start(p.q_start, p.seqs, p.total, p.status);
    for (int s = threadIdx.x; s < p.seqs; s += kThreads) {
      const int len = p.lens[s];
      if (len < 0 || len > static_cast<long long>(p.max_pages) * p.page_tokens)
        record_status(p.status, MLA_ERR_RANGE);
    }
  }
  if (threadIdx.x < 2) p.part_desc[2 * blockIdx.x + threadIdx.x] = make_int4(0, 0, 0, 0);
  const long long share =
      find_share<BN, TR>(p, blockIdx.x / CL, gridDim.x / CL, scratch, ends);
  Walk<BN, TR> walk(p, ends);
  Segment g;
  bool ok = true;
  int it = 0;  // key blocks so far: the phases of the per-block barriers
  auto phase = [](int block) { return static_cast<uint32_t>(block / NB) & 1u; };
  int sc = 0;  // ring stages so far, Q's included: the phases of kv_full, kv_empty

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
        BlockPos<BN> pos(p, g.kb0);
        auto boxes_at = [&](const BlockPos<BN>& at) {  // pages of a block that hold tokens
          const int valid = min(at.rows(p), g.st.len - at.token(p));
          return p.per_group == 1 ? (valid > 0 ? 1 : 0)
                                  : (max(valid, 0) + p.page_tokens - 1) >> page_shift;
        };
        auto look_up = [&](const BlockPos<BN>& at) {
          return lane < boxes_at(at) ? table[at.grp * p.per_group + lane] : -1;
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
        if (!ok) break;
        for (int kb = g.kb0; kb < g.kb1; ++kb, ++sc) {
          const int boxes = boxes_at(pos), sub = pos.sub, page_now = page_ahead;
          pos.step(p);
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
        for (int q = 0; q < QST; ++q, ++sc)
          if (lane < MC) {
            if constexpr (MC == 1)
              mbar_arrive(&kv_empty[sc % NST]);
            else
              mbar_arrive_cluster(dsmem_addr(smem_u32(&kv_empty[sc % NST]), lane));
          }
        BlockPos<BN> pos(p, g.kb0);
        for (int kb = g.kb0; kb < g.kb1; ++kb, ++it, ++sc, pos.step(p)) {
          const int st = sc % NST;
          uint8_t* kv = sKV + st * S::kTileBytes;
          const int valid = max(0, min(pos.rows(p), g.st.len - pos.token(p)));
          ok = __all_sync(0xffffffffu, mbar_wait(&kv_full[st], (sc / NST) & 1, wc));
          if (!ok) break;
          if (valid < BN) {
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
#pragma unroll
            for (int k = 0; k < (has_r ? DR / 16 : 0); ++k) {
              const uint64_t bd = sdesc(ka + S::kKrOff + k * 32, 16, S::kKrSbo, S::kKrSw);
              if constexpr (S::kQrTmem)
                umma_ts(d, tmem + S::kTmemQ + DV / 2 + k * 8, bd, S::kIdescQK, 1u);
              else
                umma_ss(d, sdesc(qa + S::kQKrOff + k * 32, 16, S::kKrSbo, S::kKrSw), bd,
                        S::kIdescQK, 1u);
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
      if (lane == 0) {
        while (ok && walk.next(g)) {
          sc += QST;
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
    }
  } else {
    // --------------------------------------------------- softmax (warps 4..7)
    const int quarter = warp & 3;  // TMEM lane quarter this warp may access
    const int r = quarter * 32 + lane;
    const uint32_t t_lane = static_cast<uint32_t>(quarter * 32) << 16;
    int xc = 0;  // blocks exchanged with the peer
    struct Row {
      int tile0, lrow, keys;  // the CTA's first row, this thread's, the keys it sees
      size_t grow;            // its place in q and o
      bool ok, warp_ok;       // the row exists; one of the warp's does
    };
    // The thread's row of a segment, and its Q, from the ring stage into TMEM
    // (row-major, two values a column) and shared memory (the swizzle the MMA
    // descriptors name). The score MMAs that read the previous Q are done: their
    // scores were awaited.
    auto load_row = [&](const Segment& sg, Row& w) {
      const int rows = sg.st.n * p.heads;
      w.tile0 = sg.tile * TR + first_row;
      w.lrow = w.tile0 + r;
      w.ok = w.lrow < rows;
      w.warp_ok = __any_sync(0xffffffffu, w.ok);
      w.grow = static_cast<size_t>(sg.st.q0) * p.heads + (w.ok ? w.lrow : 0);
      w.keys = w.ok ? keys_seen(p, sg.st.len - sg.st.n + p.by_heads(w.lrow), sg.st.len) : 0;
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
      tc_fence_before();
      mbar_arrive(q_ready);
      sc += QST;
      return true;
    };
    bool have = walk.next(g);
    if (!have && r == 0) p.part_desc[2 * blockIdx.x] = make_int4(0, 0, kPartEmpty, 0);
    Row w{};
    if (have) ok = load_row(g, w);
    while (ok && have) {
      float m_run = -INFINITY, l_run = 0.f;
      BlockPos<BN> pos(p, g.kb0);
      for (int kb = g.kb0; kb < g.kb1; ++kb, ++it, pos.step(p)) {
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
        const int valid = min(pos.rows(p), w.keys - pos.token(p));
        if (valid < BN) {
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
        // has none; its weights are exp2(-inf) = 0.
        float alpha = 1.f;
        bool need = false;
        if (kb == g.kb0) {
          m_run = valid > 0 ? fmaxf(m_blk, kLowest) : -INFINITY;
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
      const bool starts = g.kb0 == 0, stops = g.kb1 == g.all, whole = starts && stops;
      const int n_rows = max(0, min(kBM, g.st.n * p.heads - d.tile0));
      const int row0 = g.st.q0 * p.heads + d.tile0;
      const bool many = static_cast<long long>(g.all) * BN > kManyShares * share;
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

// Joins the partial rows of tiles that several shares cut: o = sum_k 2^(m_k - M)
// O_k over the same of l_k, in the shares' order. Every block finds the list of
// work for itself: tiles that some CTA begins and does not end. A warp takes 32 rows
// x 16 columns, a lane per row; or one row of a tile that lies row after row. Where
// many shares cut it a block takes the row, each of its warps every 16th partial
// row, unless there are many such rows.
template <int DC, int DV, int CL>
__global__ void __launch_bounds__(kJoinThreads, 1)
    paged_join_kernel(const float* part_o, const float2* part_ml, const int4* part_desc,
                      __nv_bfloat16* o, int ctas, long long out_rows) {
  constexpr int kSplit = DC / DV, kWarps = kJoinThreads / 32, kCg = DV / 4;
  constexpr int kGroups = DV / kJoinCols;
  constexpr int kV = (DV + 127) / 128;  // 4-column pieces of a row per lane
  __shared__ int4 desc[kMaxCtas];       // slots 1: tiles that begin
  __shared__ int flags[kMaxCtas];       // slots 0: what follows
  // prefix sums of the work: warps' items in the low half, blocks' in the high one
  __shared__ int items[kMaxCtas + 1];
  __shared__ int sums[8];
  __shared__ float row_m[kWarps], row_l[kWarps];
  __shared__ __align__(16) float row_o[kWarps][DV];
  grid_dep_sync();
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  int cnt = 0;
  if (threadIdx.x < ctas) {
    const int4 d = part_desc[2 * threadIdx.x + 1];
    flags[threadIdx.x] = part_desc[2 * threadIdx.x].z;
    desc[threadIdx.x] = d;
    if ((d.z & kPartHeld) && d.x >= 0 && d.y > 0 && d.y <= kBM &&
        d.x + static_cast<long long>(d.y) <= out_rows)
      cnt = d.w == 2 ? d.y << 16 : (d.w == 1 ? d.y : (d.y + 31) / 32 * kGroups);
  }
  if (warp < 5) {
#pragma unroll
    for (int s = 1; s < 32; s <<= 1) {
      const int y = __shfl_up_sync(0xffffffffu, cnt, s);
      if (lane >= s) cnt += y;
    }
    if (lane == 31) sums[warp] = cnt;
  }
  __syncthreads();
  if (warp < 5) {
    for (int w = 0; w < warp; ++w) cnt += sums[w];
    if (threadIdx.x < kMaxCtas) items[threadIdx.x + 1] = cnt;
    if (threadIdx.x == 0) items[0] = 0;
  }
  __syncthreads();
  // the tile of item `it`; sh = 0 or 16 picks the half of the prefix sums
  auto tile_of = [&](int it, int sh) {
    int lo = 0, hi = ctas - 1;
    while (lo < hi) {
      const int mid = (lo + hi + 1) / 2;
      if (((items[mid] >> sh) & 0xffff) <= it)
        lo = mid;
      else
        hi = mid - 1;
    }
    return lo;
  };
  // the chain of tile i: slot 1 of CTA i, then slot 0 of the CTAs after it in its
  // place of their pairs, up to the one that ends the tile
  auto chain_of = [&](int i) {
    for (int k0 = 1; i + k0 * CL < ctas; k0 += 32) {
      const int j = i + (k0 + lane) * CL;
      const int f = j < ctas ? flags[j] : 0;
      const unsigned stop = __ballot_sync(
          0xffffffffu, !(f & (kPartHeld | kPartEmpty)) || (f & kPartEnds));
      if (stop) {
        const int l = __ffs(stop) - 1;
        return k0 + l + ((__shfl_sync(0xffffffffu, f, l) & kPartHeld) ? 1 : 0);
      }
    }
    return (ctas - 1 - i) / CL + 1;
  };
  auto slot_of = [&](int i, int k) { return k == 0 ? 2 * i + 1 : 2 * (i + k * CL); };
  auto holds = [&](int i, int k) { return k == 0 || (flags[i + k * CL] & kPartHeld); };

  // One row of tile i, partial rows first, first + step, ... of its chain: maximum,
  // sum and the lane's columns 4 (lane + 32 c).
  auto row_part = [&](int i, int row, int n, int first, int step, float& m, float& l,
                      float4 (&acc)[kV]) {
    m = -INFINITY;
    l = 0.f;
#pragma unroll
    for (int c = 0; c < kV; ++c) acc[c] = make_float4(0.f, 0.f, 0.f, 0.f);
    for (int base = first; base < n; base += 32 * step) {
      const int k = base + lane * step;
      float2 ml = make_float2(-INFINITY, 0.f);
      if (k < n && holds(i, k)) ml = part_ml[slot_of(i, k) * kBM + row];
      const unsigned none = __ballot_sync(0xffffffffu, ml.x == -INFINITY);
      float mx = ml.x;
#pragma unroll
      for (int s = 16; s > 0; s >>= 1) mx = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, s));
      const float m_new = fmaxf(m, mx), ref = m_new == -INFINITY ? 0.f : m_new;
      const float a = ex2_approx(m - ref), w = ex2_approx(ml.x - ref);
      float wl = w * ml.y;
#pragma unroll
      for (int s = 16; s > 0; s >>= 1) wl += __shfl_xor_sync(0xffffffffu, wl, s);
      m = m_new;
      l = l * a + wl;
#pragma unroll
      for (int c = 0; c < kV; ++c) {
        acc[c].x *= a;
        acc[c].y *= a;
        acc[c].z *= a;
        acc[c].w *= a;
      }
      const int cnt = min(32, (n - base + step - 1) / step);
      // four rows at a time, all loads of a group in flight together (past the
      // chain's end the last row again, at weight 0)
#pragma unroll 1
      for (int t0 = 0; t0 < cnt; t0 += 4) {
        float4 v[4][kV];
#pragma unroll
        for (int t = 0; t < 4; ++t) {
          const float4* src = reinterpret_cast<const float4*>(
              part_o +
              (static_cast<size_t>(slot_of(i, base + min(t0 + t, cnt - 1) * step)) * kBM + row) *
                  DV);
#pragma unroll
          for (int c = 0; c < kV; ++c)
            if (lane + 32 * c < kCg) v[t][c] = src[lane + 32 * c];
        }
#pragma unroll
        for (int t = 0; t < 4; ++t) {
          const float wt = __shfl_sync(0xffffffffu, w, t0 + t);
          if (none >> (t0 + t) & 1) continue;  // an empty share's slot may hold anything
#pragma unroll
          for (int c = 0; c < kV; ++c) {
            acc[c].x += wt * v[t][c].x;
            acc[c].y += wt * v[t][c].y;
            acc[c].z += wt * v[t][c].z;
            acc[c].w += wt * v[t][c].w;
          }
        }
      }
    }
  };
  auto out_row = [&](int i, int row) {
    return o + (static_cast<size_t>(desc[i].x) + row) * DC + (kSplit > 1 ? i % CL : 0) * DV;
  };

  // More rows than two per block: a warp each (16 rows at once in a chain of a few
  // steps beat one row at once in a short one: 16 streams of 5 tokens at d_c = 512
  // 50.9 -> 46.8 us)
  const int warp_items = items[ctas] & 0xffff, rows_left = items[ctas] >> 16;
  const bool spread = rows_left > 2 * static_cast<int>(gridDim.x);
  const int warp_count = warp_items + (spread ? rows_left : 0);
  const int block_items = spread ? 0 : rows_left;
  for (int it = blockIdx.x + gridDim.x * warp; it < warp_count; it += gridDim.x * kWarps) {
    const int sh = it < warp_items ? 0 : 16, at = it < warp_items ? it : it - warp_items;
    const int i = tile_of(at, sh), n = chain_of(i);
    const int4 d = desc[i];
    const int sub = at - ((items[i] >> sh) & 0xffff);
    if (d.w != 0) {
      float m, l;
      float4 acc[kV];
      row_part(i, sub, n, 0, 1, m, l, acc);
      const float f = l == 0.f ? 0.f : 1.f / l;
#pragma unroll
      for (int c = 0; c < kV; ++c)
        if (lane + 32 * c < kCg)
          reinterpret_cast<uint2*>(out_row(i, sub))[lane + 32 * c] =
              make_uint2(pack_bf16x2(acc[c].x * f, acc[c].y * f),
                         pack_bf16x2(acc[c].z * f, acc[c].w * f));
      continue;
    }
    const int rb = sub / kGroups, cg0 = (sub - rb * kGroups) * (kJoinCols / 4);
    const int row = rb * 32 + lane;
    const bool ok = row < d.y;
    float m = -INFINITY, l = 0.f;
    float4 acc[4] = {};
    // the chain in groups of four, all loads of a group in flight together; rows
    // and slots that hold nothing are loaded and not used
#pragma unroll 1
    for (int k0 = 0; k0 < n; k0 += 4) {
      float2 ml[4];
      float4 v[4][4];
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        const int kk = min(k0 + k, n - 1), sl = slot_of(i, kk);
        ml[k] = part_ml[sl * kBM + row];
        if (!ok || k0 + k >= n || !holds(i, kk)) ml[k] = make_float2(-INFINITY, 0.f);
#pragma unroll
        for (int c = 0; c < 4; ++c)
          v[k][c] = reinterpret_cast<const float4*>(
              part_o)[(static_cast<size_t>(sl) * kCg + cg0 + c) * kBM + row];
      }
      const float m_new =
          fmaxf(fmaxf(fmaxf(ml[0].x, ml[1].x), fmaxf(ml[2].x, ml[3].x)), m);
      const float ref = m_new == -INFINITY ? 0.f : m_new;
      const float a = ex2_approx(m - ref);
      m = m_new;
      l *= a;
#pragma unroll
      for (int c = 0; c < 4; ++c) {
        acc[c].x *= a;
        acc[c].y *= a;
        acc[c].z *= a;
        acc[c].w *= a;
      }
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        const float b = ex2_approx(ml[k].x - ref);
        if (ml[k].x != -INFINITY) {
          l += ml[k].y * b;
#pragma unroll
          for (int c = 0; c < 4; ++c) {
            acc[c].x += v[k][c].x * b;
            acc[c].y += v[k][c].y * b;
            acc[c].z += v[k][c].z * b;
            acc[c].w += v[k][c].w * b;
          }
        }
      }
    }
    if (ok) {
      const float f = l == 0.f ? 0.f : 1.f / l;
      uint4* dst = reinterpret_cast<uint4*>(out_row(i, row) + cg0 * 4);
#pragma unroll
      for (int c = 0; c < 2; ++c)
        dst[c] = make_uint4(pack_bf16x2(acc[2 * c].x * f, acc[2 * c].y * f),
                            pack_bf16x2(acc[2 * c].z * f, acc[2 * c].w * f),
                            pack_bf16x2(acc[2 * c + 1].x * f, acc[2 * c + 1].y * f),
                            pack_bf16x2(acc[2 * c + 1].z * f, acc[2 * c + 1].w * f));
    }
  }

  for (int it = blockIdx.x; it < block_items; it += gridDim.x) {
    const int i = tile_of(it, 16), n = chain_of(i), row = it - (items[i] >> 16);
    float m, l;
    float4 acc[kV];
    row_part(i, row, n, warp, kWarps, m, l, acc);
#pragma unroll
    for (int c = 0; c < kV; ++c)
      if (lane + 32 * c < kCg) reinterpret_cast<float4*>(row_o[warp])[lane + 32 * c] = acc[c];
    if (lane == 0) {
      row_m[warp] = m;
      row_l[warp] = l;
    }
    __syncthreads();
    if (threadIdx.x < DV) {
      float top = row_m[0], sum = 0.f, v = 0.f;
#pragma unroll
      for (int w = 1; w < kWarps; ++w) top = fmaxf(top, row_m[w]);
      const float ref = top == -INFINITY ? 0.f : top;
#pragma unroll
      for (int w = 0; w < kWarps; ++w) {
        const float wt = ex2_approx(row_m[w] - ref);
        sum += wt * row_l[w];
        v += wt * row_o[w][threadIdx.x];
      }
      out_row(i, row)[threadIdx.x] = __float2bfloat16_rn(sum == 0.f ? v * 0.f : v / sum);
    }
    __syncthreads();  // the rows in shared memory are the next item's
  }
}

template <int DC, int DV, int CL>
int launch_join(const PagedK& k, int ctas, const PagedAttnArgs& a) {
  return launch_pdl(paged_join_kernel<DC, DV, CL>, dim3(kJoinGrid), kJoinThreads, 0, a.stream,
                    k.part_o, k.part_ml, k.part_desc, k.o, ctas,
                    static_cast<long long>(a.total) * a.heads);
}

template <int DC, int DR, int CL>
int launch_paged(const PagedAttnArgs& a) {
  using S = PagedShape<DC, DR>;
  const PagedK k = paged_params(a, S::BN, S::DV);
  CUtensorMap tm_c, tm_kr;
  const unsigned long long rows = static_cast<unsigned long long>(a.pages) * a.page_tokens;
  if (!encode_map_2d_bf16(&tm_c, a.c, DC, rows, DC * 2ull, 64, k.box_rows,
                          CU_TENSOR_MAP_SWIZZLE_128B) ||
      !encode_map_2d_bf16(&tm_kr, a.kr, DR, rows, DR * 2ull, DR, k.box_rows,
                          DR == 32 ? CU_TENSOR_MAP_SWIZZLE_64B : CU_TENSOR_MAP_SWIZZLE_128B))
    return MLA_ERR_CUDA;
  CUtensorMap tm_qc, tm_qr;  // boxes of 32 rows: short tiles fetch what they have
  const unsigned long long q_rows = static_cast<unsigned long long>(a.total) * a.heads;
  if (!encode_map_2d_bf16(&tm_qc, a.q_c, DC, q_rows, DC * 2ull, 64, 32,
                          CU_TENSOR_MAP_SWIZZLE_128B) ||
      !encode_map_2d_bf16(&tm_qr, a.q_r, DR, q_rows, DR * 2ull, DR, 32,
                          DR == 32 ? CU_TENSOR_MAP_SWIZZLE_64B : CU_TENSOR_MAP_SWIZZLE_128B))
    return MLA_ERR_CUDA;
  auto kern = paged_attn_kernel<DC, DR, CL>;
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
  const cudaError_t e = cudaLaunchKernelEx(&cfg, kern, tm_c, tm_kr, tm_qc, tm_qr, k);
  if (e != cudaSuccess) {
    (void)cudaGetLastError();
    set_last_cuda_error(e);
    return MLA_ERR_CUDA;
  }
  return launch_join<DC, S::DV, CL>(k, resident, a);
}

// Two row tiles and more a slot of the pool on average: CTA pairs, which read each key
// tile from L2 once for 256 rows. Shorter ones would leave half a pair idle (ragged
// prompts 51 us with pairs, 60 without). Idle slots count as short streams here too: a
// 4,680-token chunk on 32,760 keys 820 us in a pool of 4 slots, 891 of 256.
template <int DC, int DR>
int pick(const PagedAttnArgs& a) {
  if constexpr (PagedShape<DC, DR>::kSplit == 2) {
    return launch_paged<DC, DR, 2>(a);
  } else {
    return static_cast<long long>(a.total) * a.heads >= 2ll * kBM * a.seqs
               ? launch_paged<DC, DR, 2>(a)
               : launch_paged<DC, DR, 1>(a);
  }
}

template <int DR>
int pick_dc(const PagedAttnArgs& a) {
  switch (a.d_c) {
    case 64: return pick<64, DR>(a);
    case 128: return pick<128, DR>(a);
    case 192: return pick<192, DR>(a);
    case 256: return pick<256, DR>(a);
    case 512: return pick<512, DR>(a);
    default: return MLA_ERR_UNSUPPORTED;
  }
}

}  // namespace

unsigned long long paged_attention_workspace(int d_c, int d_r) {
  if (d_r != 32 && d_r != 64) return 0;
  switch (d_c) {
    case 64:
    case 128:
    case 192:
    case 256: return PartLayout(d_c).total;
    case 512: return PartLayout(256).total;
    default: return 0;
  }
}

int launch_paged_join(const PagedK& k, int ctas, const PagedAttnArgs& a) {
  switch (a.d_c) {
    case 64: return launch_join<64, 64, 1>(k, ctas, a);
    case 128: return launch_join<128, 128, 1>(k, ctas, a);
    case 192: return launch_join<192, 192, 1>(k, ctas, a);
    case 256: return launch_join<256, 256, 1>(k, ctas, a);
    default: return MLA_ERR_UNSUPPORTED;
  }
}

int launch_paged_attention(const PagedAttnArgs& a) {
  // Up to 16 rows a slot of the pool on average, as one token of 8 to 16 heads of every
  // stream: the kernel of 16-row tiles (13.3 -> 11.2 us for one token when it was added).
  // The host knows the slots and the rows, not which streams have them: a few streams'
  // chunks in a pool of many idle slots come here too and are slower than in a small pool
  // (333 tokens on 5,001 keys, 12 heads: 29 us in a pool of 4 slots, 34 of 64, 105 of 256,
  // 187 of 1,024).
  if (a.d_c <= 256 && static_cast<long long>(a.total) * a.heads <= 16ll * a.seqs)
    return launch_paged_decode(a);
  return a.d_r == 32 ? pick_dc<32>(a) : pick_dc<64>(a);
}

}  // namespace vmla
