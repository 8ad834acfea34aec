// Attention of ragged streams' newest tokens over a paged latent cache (Eq.
// score; App. E): one block per (token, head) row, keys in tiles of 128 with a
// running maximum and sum (fp32).
#include <cmath>

#include "internal.h"
#include "paged_common.cuh"
#include "ptx_sm103.cuh"

namespace vmla {
namespace {

constexpr int kThreads = 128;
constexpr int kMaxDC = 512, kMaxDR = 64;

__device__ __forceinline__ float block_reduce(float v, float* red, bool is_max) {
#pragma unroll
  for (int d = 16; d > 0; d >>= 1) {
    const float w = __shfl_xor_sync(0xffffffffu, v, d);
    v = is_max ? fmaxf(v, w) : v + w;
  }
  __syncthreads();
  if ((threadIdx.x & 31) == 0) red[threadIdx.x >> 5] = v;
  __syncthreads();
  return is_max ? fmaxf(fmaxf(red[0], red[1]), fmaxf(red[2], red[3]))
                : (red[0] + red[1]) + (red[2] + red[3]);
}

__device__ __forceinline__ float dot8(uint4 v, const float* q) {
  return bf16_lo(v.x) * q[0] + bf16_hi(v.x) * q[1] + bf16_lo(v.y) * q[2] + bf16_hi(v.y) * q[3] +
         bf16_lo(v.z) * q[4] + bf16_hi(v.z) * q[5] + bf16_lo(v.w) * q[6] + bf16_hi(v.w) * q[7];
}

__global__ void __launch_bounds__(kThreads) paged_attn_simple_kernel(const PagedAttnArgs p) {
  grid_dep_sync();
  __shared__ float q[kMaxDC + kMaxDR], w[kThreads], red[4];
  __shared__ int pages[kThreads];
  if (blockIdx.x == 0) check_q_start(p.q_start, p.seqs, p.total, p.status);
  const __nv_bfloat16* c = static_cast<const __nv_bfloat16*>(p.c);
  const int t = blockIdx.x / p.heads;
  const int s = stream_of(p.q_start, p.seqs, t, threadIdx.x & 31);
  const int q0 = p.q_start[s], q1 = p.q_start[s + 1], len = p.lens[s];
  if (t < q0 || t >= q1 || q0 < 0 || q1 > p.total || len < 0 ||
      len > static_cast<long long>(p.max_pages) * p.page_tokens) {
    if (threadIdx.x == 0) record_status(p.status, MLA_ERR_RANGE);
    return;
  }
  const int keys = visible_keys(len - (q1 - q0) + (t - q0), len, p.causal_block);
  const size_t row = blockIdx.x;
  for (int i = threadIdx.x; i < p.d_c; i += kThreads)
    q[i] = __bfloat162float(static_cast<const __nv_bfloat16*>(p.q_c)[row * p.d_c + i]);
  for (int i = threadIdx.x; i < p.d_r; i += kThreads)
    q[p.d_c + i] = __bfloat162float(static_cast<const __nv_bfloat16*>(p.q_r)[row * p.d_r + i]);
  float m = -INFINITY, l = 0.f, o[kMaxDC / kThreads] = {};
  for (int k0 = 0; k0 < keys; k0 += kThreads) {
    __syncthreads();
    const int k = k0 + threadIdx.x;
    int page = -1;
    if (k < keys) {
      page = p.table[static_cast<size_t>(s) * p.max_pages + k / p.page_tokens];
      if (page < 0 || page >= p.pages) {
        record_status(p.status, MLA_ERR_RANGE);
        page = -1;
      }
    }
    pages[threadIdx.x] = page;
    float sc = 0.f;
    if (page >= 0) {
      const size_t r = static_cast<size_t>(page) * p.page_tokens + k % p.page_tokens;
      const uint4* cr = static_cast<const uint4*>(p.c) + r * (p.d_c / 8);
      const uint4* kr = static_cast<const uint4*>(p.kr) + r * (p.d_r / 8);
      for (int i = 0; i < p.d_c / 8; ++i) sc += dot8(__ldg(cr + i), q + 8 * i);
      for (int i = 0; i < p.d_r / 8; ++i) sc += dot8(__ldg(kr + i), q + p.d_c + 8 * i);
    }
    sc = k < keys ? sc * p.scale_log2 : -INFINITY;
    const float m_new = fmaxf(m, block_reduce(sc, red, true));
    const float base = m_new == -INFINITY ? 0.f : m_new;
    const float e = exp2f(sc - base), alpha = exp2f(m - base);
    w[threadIdx.x] = e;
    l = l * alpha + block_reduce(e, red, false);
    m = m_new;
    const int n = min(kThreads, keys - k0);
#pragma unroll
    for (int i = 0; i < kMaxDC / kThreads; ++i) {
      const int col = threadIdx.x + i * kThreads;
      if (col >= p.d_c) break;
      float acc = o[i] * alpha;
      for (int j = 0; j < n; ++j)
        if (pages[j] >= 0)
          acc += w[j] * __bfloat162float(
                            c[(static_cast<size_t>(pages[j]) * p.page_tokens +
                               (k0 + j) % p.page_tokens) * p.d_c + col]);
      o[i] = acc;
    }
  }
  const float inv = l > 0.f ? 1.f / l : (l == 0.f ? 0.f : l);  // a NaN stays one
#pragma unroll
  for (int i = 0; i < kMaxDC / kThreads; ++i) {
    const int col = threadIdx.x + i * kThreads;
    if (col < p.d_c)
      static_cast<__nv_bfloat16*>(p.o)[row * p.d_c + col] = __float2bfloat16_rn(o[i] * inv);
  }
}

}  // namespace

unsigned long long paged_attention_workspace(int d_c, int d_r) {
  const bool ok = (d_c == 64 || d_c == 128 || d_c == 192 || d_c == 256 || d_c == 512) &&
                  (d_r == 32 || d_r == 64);
  return ok ? 16 : 0;
}

int launch_paged_attention(const PagedAttnArgs& a) {
  return launch_pdl(paged_attn_simple_kernel, dim3(a.total * a.heads), kThreads, 0, a.stream, a);
}

}  // namespace vmla
