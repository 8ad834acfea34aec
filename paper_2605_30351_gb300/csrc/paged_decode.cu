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
#include <cmath>

#include "internal.h"
#include "paged_attn.cuh"
#include "ptx_sm103.cuh"

namespace vmla {
namespace {

constexpr int kWarps = 8;
constexpr int kThreads = 32 * kWarps;
constexpr int kRows = 16;                     // rows of a tile
constexpr int kBN = 16 * kWarps;              // keys of a block
constexpr float kRescaleLog2 = 8.0f;
constexpr int kRedStride = 40;                // floats per row of a reduction tile (32 + pad)

template <int DC, int DR>
struct DecodeShape {
  static constexpr int DK = DC + DR;
  static constexpr int kTileBytes = 16 * DK * 2;  // a warp's stage of 16 keys:
  static constexpr int kCBox = 16 * 128;          // [16 x 64 columns] of c each,
  static constexpr int kKrOff = DC * 16 * 2;      // then the d_r columns
  static constexpr int kKrRow = DR * 2;
  static constexpr int kQStride = DK * 2 + 16;  // bytes; rows in different banks
  static constexpr int kQBytes = kRows * kQStride;
  static constexpr int kRedBytes = 2 * kWarps * kRows * kRedStride * 4;
  static constexpr int kMlBytes = kWarps * kRows * 8;
  static constexpr int kRest = 1024 + kQBytes + kRedBytes + kMlBytes + 128;
  static constexpr int kFit = (232448 - kRest) / (kTileBytes * kWarps);
  static constexpr int kStages = kFit > 4 ? 4 : kFit;
  static constexpr int kSmemBytes = kRest + kTileBytes * kWarps * kStages;
  static constexpr bool kQRegs = DC <= 192;
  static_assert(kStages >= 2 && kQBytes % 16 == 0, "two stages must fit");
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

template <int DC, int DR>
__global__ void __launch_bounds__(kThreads, 1)
    paged_decode_kernel(const uint8_t* c, const uint8_t* kr, const __nv_bfloat16* q_c,
                        const __nv_bfloat16* q_r, const PagedK p) {
  using S = DecodeShape<DC, DR>;
  constexpr int NST = S::kStages, kSteps = S::DK / 16;
  extern __shared__ uint8_t smem_raw[];
  uint8_t* sKV = align_smem_1024(smem_raw);
  uint8_t* sQ = sKV + NST * kWarps * S::kTileBytes;
  float* red = reinterpret_cast<float*>(sQ + S::kQBytes);  // [2][warps][16][kRedStride]
  float2* warp_ml = reinterpret_cast<float2*>(red + 2 * kWarps * kRows * kRedStride);
  long long* scratch = reinterpret_cast<long long*>(warp_ml + kWarps * kRows);  // [8]
  Place* ends = reinterpret_cast<Place*>(scratch + 8);                          // [2]

  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  grid_dep_sync();
  if (blockIdx.x == 0) {
    check_q_start(p.q_start, p.seqs, p.total, p.status);
    for (int s = threadIdx.x; s < p.seqs; s += kThreads) {
      const int len = p.lens[s];
      if (len < 0 || len > static_cast<long long>(p.max_pages) * p.page_tokens)
        record_status(p.status, MLA_ERR_RANGE);
    }
  }
  if (threadIdx.x < 2) p.part_desc[2 * blockIdx.x + threadIdx.x] = make_int4(0, 0, 0, 0);
  find_share<kBN, kRows>(p, blockIdx.x, gridDim.x, scratch, ends);
  Walk<kBN, kRows> walk(p, ends);
  Segment g;
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
  while (walk.next(g)) {
    any = true;
    const int rows = g.st.n * p.heads, row0 = g.tile * kRows;
    const int n_rows = min(kRows, rows - row0);
    const size_t grow = static_cast<size_t>(g.st.q0) * p.heads + row0;
    constexpr int kPc = DC / 8, kPr = DR / 8;  // 16-byte pieces of a row
    for (int i = threadIdx.x; i < kRows * (kPc + kPr); i += kThreads) {
      const int r = i / (kPc + kPr), pc = i - r * (kPc + kPr);
      uint4 v = make_uint4(0u, 0u, 0u, 0u);
      if (r < n_rows)
        v = pc < kPc
                ? reinterpret_cast<const uint4*>(q_c + (grow + r) * DC)[pc]
                : reinterpret_cast<const uint4*>(q_r + (grow + r) * DR)[pc - kPc];
      *reinterpret_cast<uint4*>(sQ + r * S::kQStride + pc * 16) = v;
    }
    auto keys_of = [&](int r) {
      return r < n_rows
                 ? keys_seen(p, g.st.len - g.st.n + p.by_heads(row0 + r), g.st.len)
                 : 0;
    };
    const int keys_a = keys_of(ra), keys_b = keys_of(rb);

    // The ring: block kb0 + i goes to stage i % NST, NST - 1 blocks ahead of the one
    // that is computed. The pages of the next block to fetch are looked up one
    // block ahead of that.
    const int n_blocks = g.kb1 - g.kb0;
    const int* table = p.table + static_cast<size_t>(g.s) * p.max_pages;
    BlockPos<kBN> ahead(p, g.kb0);
    int page_a = -1, page_b = -1;
    auto held = [&](const BlockPos<kBN>& at) {  // tokens among the warp's 16 keys
      return min(at.rows(p) - 16 * warp, g.st.len - at.token(p) - 16 * warp);
    };
    auto look_up = [&](int i) {
      if (i < n_blocks && held(ahead) > 0) {
        const int at = ahead.grp * p.per_group + page_at;
        page_a = table[at];
        page_b = page_step && held(ahead) > 8 ? table[at + 1] : page_a;
      }
    };
    auto fetch = [&](int i) {
      const int n = i < n_blocks ? held(ahead) : 0;
      if (n > 0) {
        if (page_a < 0 || page_a >= p.pages || page_b < 0 || page_b >= p.pages)
          record_status(p.status, MLA_ERR_RANGE);
        const uint32_t dst = ring + (i % NST) * S::kTileBytes;
        const int off = ahead.sub * kBN + off_at;
#pragma unroll
        for (int rg = 0; rg < 4; ++rg) {  // 4 rows x 128 bytes of c at a time
          const int row = 4 * rg + (lane >> 3), pc = lane & 7;
          const int page = row < 8 ? page_a : page_b;
          const bool in = row < n && page >= 0 && page < p.pages;
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
          const bool in = row < n && page >= 0 && page < p.pages;
          const size_t at = in ? static_cast<size_t>(page) * p.page_tokens + off + row -
                                     (page_step && row >= 8 ? 8 : 0)
                               : 0;
          const int sw = DR == 32 ? (row >> 1) & 3 : row & 7;
          copy16(dst + S::kKrOff + row * S::kKrRow + ((pc ^ sw) * 16),
                 kr + at * (DR * 2) + pc * 16, in ? 16 : 0);
        }
      }
      asm volatile("cp.async.commit_group;" ::: "memory");
      ahead.step(p);
      look_up(i + 1);
    };
    look_up(0);
#pragma unroll 1
    for (int i = 0; i < NST - 1; ++i) fetch(i);
    __syncthreads();
    uint32_t q[S::kQRegs ? kSteps : 1][4];
    if constexpr (S::kQRegs) {
#pragma unroll
      for (int k = 0; k < kSteps; ++k) ldm4(q[k], q_at + k * 32);
    }
    float o[DC / 8][4];
#pragma unroll
    for (int i = 0; i < DC / 8; ++i)
#pragma unroll
      for (int c = 0; c < 4; ++c) o[i][c] = 0.f;
    float m_a = -INFINITY, m_b = -INFINITY, l_a = 0.f, l_b = 0.f;

    BlockPos<kBN> pos(p, g.kb0);
#pragma unroll 1
    for (int i = 0; i < n_blocks; ++i, pos.step(p)) {
      fetch(i + NST - 1);
      asm volatile("cp.async.wait_group %0;" ::"n"(NST - 1) : "memory");
      __syncwarp();
      const int token = pos.token(p) + 16 * warp, room = pos.rows(p) - 16 * warp;
      if (held(pos) > 0) {
        const uint32_t ka = ring + (i % NST) * S::kTileBytes;
        float s[2][4];  // two tiles of 8 keys
#pragma unroll
        for (int i = 0; i < 2; ++i)
#pragma unroll
          for (int c = 0; c < 4; ++c) s[i][c] = 0.f;
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
            ldm4(q[0], q_at + k * 32);
            mma16816(s[0], q[0], b[0], b[1]);
            mma16816(s[1], q[0], b[2], b[3]);
          }
        }
        const int lim_a = min(room, keys_a - token), lim_b = min(room, keys_b - token);
#pragma unroll
        for (int i = 0; i < 2; ++i)
#pragma unroll
          for (int c = 0; c < 2; ++c) {
            const int key = 8 * i + cq + c;
            if (key >= lim_a) s[i][c] = -INFINITY;
            if (key >= lim_b) s[i][2 + c] = -INFINITY;
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
        const bool up_a = x_a > m_a + kRescaleLog2 || (m_a == -INFINITY && x_a > m_a);
        const bool up_b = x_b > m_b + kRescaleLog2 || (m_b == -INFINITY && x_b > m_b);
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
    const bool whole = g.kb0 == 0 && g.kb1 == g.all;
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
#pragma unroll
    for (int c = 0; c < DC / 32; ++c) {  // 32 columns at a time, two buffers
      float* buf = red + (c & 1) * kWarps * kRows * kRedStride;
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        float* at = buf + (warp * kRows + ra) * kRedStride + 8 * i + cq;
        const float(&v)[4] = o[4 * c + i];
        *reinterpret_cast<float2*>(at) = make_float2(v[0] * f_a, v[1] * f_a);
        *reinterpret_cast<float2*>(at + 8 * kRedStride) = make_float2(v[2] * f_b, v[3] * f_b);
      }
      __syncthreads();
      float2 sum = make_float2(0.f, 0.f);
#pragma unroll
      for (int w = 0; w < kWarps; ++w) {
        const float2 v =
            *reinterpret_cast<const float2*>(buf + (w * kRows + out_r) * kRedStride + out_c);
        sum.x += v.x;
        sum.y += v.y;
      }
      if (out_r < n_rows) {
        if (whole)
          *reinterpret_cast<uint32_t*>(p.o + (grow + out_r) * DC + 32 * c + out_c) =
              pack_bf16x2(sum.x, sum.y);
        else
          *reinterpret_cast<float2*>(p.part_o + (static_cast<size_t>(slot) * kBM + out_r) * DC +
                                     32 * c + out_c) = sum;
      }
    }
    if (!whole && threadIdx.x < n_rows) {
      float2 t = total_of(threadIdx.x);
      if (keys_of(threadIdx.x) > BlockPos<kBN>(p, g.kb0).token(p)) t.x = fmaxf(t.x, kLowest);
      p.part_ml[slot * kBM + threadIdx.x] = t;
    }
    if (!whole && threadIdx.x == 0)
      p.part_desc[slot] = make_int4(static_cast<int>(grow), n_rows,
                                    kPartHeld | (g.kb1 == g.all ? kPartEnds : 0), 2);
    __syncthreads();  // sQ, the sums and the buffers are the next segment's
  }
  if (!any && threadIdx.x == 0)
    p.part_desc[2 * blockIdx.x] = make_int4(0, 0, kPartEmpty, 0);
}

template <int DC, int DR>
int launch_decode(const PagedAttnArgs& a) {
  using S = DecodeShape<DC, DR>;
  const PagedK k = paged_params(a, kBN, DC);
  auto kern = paged_decode_kernel<DC, DR>;
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
  const int rc = launch_pdl(kern, dim3(ctas), kThreads, S::kSmemBytes, a.stream,
                            static_cast<const uint8_t*>(a.c), static_cast<const uint8_t*>(a.kr),
                            static_cast<const __nv_bfloat16*>(a.q_c),
                            static_cast<const __nv_bfloat16*>(a.q_r), k);
  return rc != MLA_OK ? rc : launch_paged_join(k, ctas, a);
}

template <int DR>
int pick(const PagedAttnArgs& a) {
  switch (a.d_c) {
    case 64: return launch_decode<64, DR>(a);
    case 128: return launch_decode<128, DR>(a);
    case 192: return launch_decode<192, DR>(a);
    case 256: return launch_decode<256, DR>(a);
    default: return MLA_ERR_UNSUPPORTED;
  }
}

}  // namespace

int launch_paged_decode(const PagedAttnArgs& a) {
  return a.d_r == 32 ? pick<32>(a) : pick<64>(a);
}

}  // namespace vmla
