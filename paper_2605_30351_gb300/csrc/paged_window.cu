// Attention of ragged streams' newest tokens over the sinks and the sliding window of a
// paged latent cache (Eq. score; App. D.4, D.5, E): a simple kernel, one block for each
// (token, head) row, one warp for each key in turn.
#include <cmath>

#include "internal.h"
#include "paged_attn.cuh"
#include "ptx_sm103.cuh"

namespace vmla {
namespace {

constexpr int kThreads = 128;
constexpr int kWarps = kThreads / 32;

template <int DC, int DR>
__global__ void __launch_bounds__(kThreads)
    window_simple_kernel(const PagedAttnArgs a) {
  __shared__ float ml[kWarps][2];
  __shared__ float acc[kWarps][DC];
  grid_dep_sync();
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const int t = blockIdx.x / a.heads;
  if (blockIdx.x == 0) check_q_start(a.q_start, a.seqs, a.total, a.status);
  const int s = stream_of(a.q_start, a.seqs, t, lane);
  const int q0 = a.q_start[s], q1 = a.q_start[s + 1], len = a.lens[s];
  const int gone = a.dropped ? a.dropped[s] : 0;
  const long long front =
      (static_cast<long long>(a.sinks) + a.page_tokens - 1) / a.page_tokens * a.page_tokens;
  if (len < 0 || len > static_cast<long long>(a.max_pages) * a.page_tokens || gone < 0 ||
      static_cast<long long>(len) + gone >= kMostTokens ||
      (gone > 0 && len - static_cast<long long>(q1 - q0) < front)) {
    if (threadIdx.x == 0) record_status(a.status, MLA_ERR_RANGE);
    return;
  }
  if (t < q0 || t >= q1 || q1 > a.total) return;
  // keys: places [0, sink_end) and [low, end)
  const long long place = static_cast<long long>(len) - (q1 - q0) + (t - q0);
  long long end = 0, sink_end = 0, low = 0;
  if (place >= 0) {
    end = len;
    if (a.causal_block > 0)
      end = min(end, ((place + gone) / a.causal_block + 1) * a.causal_block - gone);
    sink_end = min(end, static_cast<long long>(a.sinks));
    low = max(gone > 0 ? front : static_cast<long long>(a.sinks), end - a.window);
  }
  const size_t row = static_cast<size_t>(blockIdx.x);
  const __nv_bfloat16* q_c = static_cast<const __nv_bfloat16*>(a.q_c) + row * DC;
  const __nv_bfloat16* q_r = static_cast<const __nv_bfloat16*>(a.q_r) + row * DR;
  const __nv_bfloat16* q_s =
      a.q_sink ? static_cast<const __nv_bfloat16*>(a.q_sink) + row * DR : q_r;
  const __nv_bfloat16* c = static_cast<const __nv_bfloat16*>(a.c);
  const __nv_bfloat16* kr = static_cast<const __nv_bfloat16*>(a.kr);
  float m = -INFINITY, l = 0.f, o[DC / 32] = {};
  const long long keys = sink_end + max(0ll, end - low);
  for (long long k = warp; k < keys; k += kWarps) {
    const long long j = k < sink_end ? k : low + (k - sink_end);
    const int page = a.table[static_cast<size_t>(s) * a.max_pages + j / a.page_tokens];
    const bool in = page >= 0 && page < a.pages;
    if (!in && lane == 0) record_status(a.status, MLA_ERR_RANGE);
    const size_t at = in ? static_cast<size_t>(page) * a.page_tokens + j % a.page_tokens : 0;
    const __nv_bfloat16* q = k < sink_end ? q_s : q_r;
    float v[DC / 32], x = 0.f;
#pragma unroll
    for (int i = 0; i < DC / 32; ++i) {
      v[i] = in ? __bfloat162float(c[at * DC + i * 32 + lane]) : 0.f;
      x += __bfloat162float(q_c[i * 32 + lane]) * v[i];
    }
#pragma unroll
    for (int i = 0; i < DR / 32; ++i)
      x += __bfloat162float(q[i * 32 + lane]) *
           (in ? __bfloat162float(kr[at * DR + i * 32 + lane]) : 0.f);
#pragma unroll
    for (int d = 16; d > 0; d >>= 1) x += __shfl_xor_sync(0xffffffffu, x, d);
    x *= a.scale_log2;
    const float m_new = fmaxf(fmaxf(m, x), kLowest);
    const float f = ex2_approx(m - m_new), w = ex2_approx(x - m_new);
    m = m_new;
    l = l * f + w;
#pragma unroll
    for (int i = 0; i < DC / 32; ++i) o[i] = o[i] * f + w * v[i];
  }
#pragma unroll
  for (int i = 0; i < DC / 32; ++i) acc[warp][i * 32 + lane] = o[i];
  if (lane == 0) {
    ml[warp][0] = m;
    ml[warp][1] = l;
  }
  __syncthreads();
  float top = -INFINITY;
  for (int w = 0; w < kWarps; ++w) top = fmaxf(top, ml[w][0]);
  for (int i = threadIdx.x; i < DC; i += kThreads) {
    float sum = 0.f, y = 0.f;
    for (int w = 0; w < kWarps; ++w)
      if (ml[w][0] != -INFINITY) {
        const float f = ex2_approx(ml[w][0] - top);
        sum += f * ml[w][1];
        y += f * acc[w][i];
      }
    static_cast<__nv_bfloat16*>(a.o)[row * DC + i] =
        __float2bfloat16_rn(sum == 0.f ? y * 0.f : y / sum);
  }
}

template <int DC, int DR>
int launch(const PagedAttnArgs& a) {
  return launch_pdl(window_simple_kernel<DC, DR>, dim3(a.total * a.heads), kThreads, 0, a.stream,
                    a);
}

template <int DR>
int pick(const PagedAttnArgs& a) {
  switch (a.d_c) {
    case 64: return launch<64, DR>(a);
    case 128: return launch<128, DR>(a);
    case 192: return launch<192, DR>(a);
    case 256: return launch<256, DR>(a);
    case 512: return launch<512, DR>(a);
    default: return MLA_ERR_UNSUPPORTED;
  }
}

}  // namespace

int launch_paged_window_attention(const PagedAttnArgs& a) {
  return a.d_r == 32 ? pick<32>(a) : pick<64>(a);
}

}  // namespace vmla
