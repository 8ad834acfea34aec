// New tokens of ragged streams into their pages (App. D.4), with the positional
// key rotated on the way (Sec. 3.2).
//
// One warp per token: it finds the token's stream in q_start with a 32-way
// search (one load where there are up to 32 streams), then moves the row of d_c +
// d_r values in 16-byte pieces that were fetched meanwhile. Bound by latency: q_start
// and lens, then the page table, then the store follow one another, for each token
// anew. Measured on the GPU (in a CUDA graph): 64 streams' tokens 2.6 us, 18,720 tokens
// 7.5 us (19.4 MB; the warps, of 48 and 62 registers, take two rounds; held to 32
// registers 9.9 us, to 64 7.6 us). A call from Python takes 7 us at the least: the host.
#include "internal.h"
#include "paged_common.cuh"
#include "ptx_sm103.cuh"

namespace vmla {
namespace {

constexpr int kThreads = 256;

struct AppendK {
  const uint4* c_new;
  const __nv_bfloat16* kr_new;
  const int* q_start;
  const int* pos;
  uint4* c;
  __nv_bfloat16* kr;
  const int* table;
  const int* lens;
  const float2* rope;
  int total, seqs, pages, page_tokens, max_pages, d_c, d_r;
  int rope_len, pairs_t, pairs_h, axes;
  int* status;
};

template <bool HALF>
__global__ void __launch_bounds__(kThreads) paged_append_kernel(const AppendK p) {
  grid_dep_sync();
  if (blockIdx.x == 0) check_q_start(p.q_start, p.seqs, p.total, p.status);
  const int lane = threadIdx.x & 31;
  const int warps = gridDim.x * (kThreads / 32);
  const int c16 = p.d_c / 8, m = p.d_r / 2;
  for (int t = blockIdx.x * (kThreads / 32) + (threadIdx.x >> 5); t < p.total; t += warps) {
    // the row's first pieces and the first pair's angle are on their way while
    // the token's place is found
    const uint4* src = p.c_new + static_cast<size_t>(t) * c16;
    const __nv_bfloat16* x = p.kr_new + static_cast<size_t>(t) * p.d_r;
    uint4 v = make_uint4(0u, 0u, 0u, 0u);
    if (lane < c16) v = src[lane];
    auto angle = [&](int i) {
      const int axis = p.axes == 1 || i < p.pairs_t ? 0 : (i < p.pairs_t + p.pairs_h ? 1 : 2);
      int co = p.pos[static_cast<size_t>(t) * p.axes + axis];
      if (co < 0 || co >= p.rope_len) {
        record_status(p.status, MLA_ERR_RANGE);
        co = 0;
      }
      return p.rope[static_cast<size_t>(co) * m + i];
    };
    float2 cs = make_float2(0.f, 0.f);
    float a = 0.f, b = 0.f;
    if (lane < m) {
      cs = angle(lane);
      a = __bfloat162float(x[HALF ? lane : 2 * lane]);
      b = __bfloat162float(x[HALF ? lane + m : 2 * lane + 1]);
    }
    int s, q0, q1, len;
    if (p.seqs <= 32) {  // every stream's numbers in one load, a lane per stream
      const int q = lane <= p.seqs ? p.q_start[min(lane, p.seqs)] : 0;
      const int n = lane < p.seqs ? p.lens[lane] : 0;
      const unsigned le = __ballot_sync(0xffffffffu, lane < p.seqs && q <= t);
      s = le ? 31 - __clz(le) : 0;
      q0 = __shfl_sync(0xffffffffu, q, s);
      q1 = s == 31 ? p.q_start[32] : __shfl_sync(0xffffffffu, q, (s + 1) & 31);
      len = __shfl_sync(0xffffffffu, n, s);
    } else {
      s = stream_of(p.q_start, p.seqs, t, lane);
      q0 = p.q_start[s];
      q1 = p.q_start[s + 1];
      len = p.lens[s];
    }
    const long long place = static_cast<long long>(len) - (q1 - q0) + (t - q0);
    const long long j = place / p.page_tokens;
    int page = -1;
    if (t >= q0 && t < q1 && q1 <= p.total && place >= 0 && j < p.max_pages)
      page = p.table[static_cast<size_t>(s) * p.max_pages + j];
    if (page < 0 || page >= p.pages) {
      if (lane == 0) record_status(p.status, MLA_ERR_RANGE);
      continue;
    }
    const size_t row = static_cast<size_t>(page) * p.page_tokens + (place - j * p.page_tokens);
    uint4* dst = p.c + row * c16;
    if (lane < c16) dst[lane] = v;
    for (int i = lane + 32; i < c16; i += 32) dst[i] = src[i];
    __nv_bfloat16* y = p.kr + row * p.d_r;
    for (int i = lane; i < m; i += 32) {
      const int ia = HALF ? i : 2 * i, ib = HALF ? i + m : 2 * i + 1;
      if (i != lane) {
        cs = angle(i);
        a = __bfloat162float(x[ia]);
        b = __bfloat162float(x[ib]);
      }
      y[ia] = __float2bfloat16_rn(a * cs.x - b * cs.y);
      y[ib] = __float2bfloat16_rn(a * cs.y + b * cs.x);
    }
  }
}

}  // namespace

int launch_paged_append(const PagedAppendArgs& a) {
  AppendK k;
  k.c_new = static_cast<const uint4*>(a.c_new);
  k.kr_new = static_cast<const __nv_bfloat16*>(a.kr_new);
  k.q_start = a.q_start;
  k.pos = a.pos;
  k.c = static_cast<uint4*>(a.c);
  k.kr = static_cast<__nv_bfloat16*>(a.kr);
  k.table = a.table;
  k.lens = a.lens;
  k.rope = a.rope;
  k.total = a.total;
  k.seqs = a.seqs;
  k.pages = a.pages;
  k.page_tokens = a.page_tokens;
  k.max_pages = a.max_pages;
  k.d_c = a.d_c;
  k.d_r = a.d_r;
  k.rope_len = a.rope_len;
  k.pairs_t = a.pairs_t;
  k.pairs_h = a.pairs_h;
  k.axes = a.axes;
  k.status = a.status;
  const int want = (a.total - 1) / (kThreads / 32) + 1;
  const int blocks = want < 152 * 8 ? want : 152 * 8;
  return launch_pdl(a.layout == MLA_ROPE_HALF ? paged_append_kernel<true>
                                              : paged_append_kernel<false>,
                    dim3(blocks), kThreads, 0, a.stream, k);
}

}  // namespace vmla
