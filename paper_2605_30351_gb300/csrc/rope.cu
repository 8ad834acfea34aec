// Rotary positions as an operator of their own (Sec. 3.2, App. D.3): every
// pair (a, b) of the rotated channels becomes (a cos - b sin, a sin + b cos),
// in fp32, rounded once to the tensor's type; the angles' cosines and sines
// come from a table that the host filled in double. The inverse rotation takes
// -sin.
//
// Bound by memory: each value is read once and written once, the table's 8
// bytes a (token, pair) are shared by all heads of a token. A thread takes one
// 16-byte piece (half layout: the two pieces that pair up) of kHeads heads of a
// token: its cosines and sines are fetched once for all of them, and kHeads
// loads are in flight at once. Measured on the GPU: 18,720 tokens x 12 heads x 128
// channels of bf16, the last 32 of them turned, 20.7 us (117.6 MB, 5.67 TB/s of a
// measured copy rate of 6.77); 9,999 x 16 x 128 fp32, half layout, inverse, 29.2 us
// (5.69 TB/s).
// Two heads a thread (22.1 and 29.5 us) or registers held to 48 for more warps (28.0
// and 39.1 us) were slower. Tensors whose rows or rotated part do not lie on
// 16-byte boundaries take the kernel that moves single values.
#include <cmath>

#include <cuda_fp16.h>

#include "internal.h"
#include "ptx_sm103.cuh"

namespace vmla {
namespace {

constexpr int kThreads = 256;

struct RopeK {
  const void* x;
  const int* pos;
  void* y;
  const float2* table;
  long long tokens, x_tok, x_head, y_tok, y_head;
  int heads, head_dim, table_len, pairs, pairs_t, pairs_h, axes, offset;
  float sign;
  int in_place;
  int* status;
};

__device__ __forceinline__ float to_f(float v) { return v; }
__device__ __forceinline__ float to_f(__half v) { return __half2float(v); }
__device__ __forceinline__ float to_f(__nv_bfloat16 v) { return __bfloat162float(v); }
__device__ __forceinline__ void from_f(float v, float& o) { o = v; }
__device__ __forceinline__ void from_f(float v, __half& o) { o = __float2half_rn(v); }
__device__ __forceinline__ void from_f(float v, __nv_bfloat16& o) { o = __float2bfloat16_rn(v); }

// (cos, +-sin) of pair i of a token. Plain loads: a previous kernel that still runs when
// this one starts may have written the positions.
__device__ __forceinline__ float2 pair_cs(const RopeK& p, long long t, int i) {
  const int axis = p.axes == 1 || i < p.pairs_t ? 0 : (i < p.pairs_t + p.pairs_h ? 1 : 2);
  int c = p.pos[t * p.axes + axis];
  if (c < 0 || c >= p.table_len) {
    record_status(p.status, MLA_ERR_RANGE);
    c = 0;
  }
  float2 cs = p.table[static_cast<size_t>(c) * p.pairs + i];
  cs.y *= p.sign;
  return cs;
}

// Any strides and alignment: one thread per (token, head, pair or copied channel).
template <typename T, bool HALF>
__global__ void __launch_bounds__(kThreads) rope_kernel(const RopeK p) {
  grid_dep_sync();
  const int copies = p.in_place ? 0 : p.head_dim - 2 * p.pairs;
  const int items = p.pairs + copies;
  const long long n = p.tokens * p.heads * items;
  for (long long k = blockIdx.x * static_cast<long long>(kThreads) + threadIdx.x; k < n;
       k += static_cast<long long>(gridDim.x) * kThreads) {
    const int i = static_cast<int>(k % items);
    const long long th = k / items;
    const int h = static_cast<int>(th % p.heads);
    const long long t = th / p.heads;
    const T* x = static_cast<const T*>(p.x) + t * p.x_tok + h * p.x_head;
    T* y = static_cast<T*>(p.y) + t * p.y_tok + h * p.y_head;
    if (i < p.pairs) {
      const float2 cs = pair_cs(p, t, i);
      const int ia = p.offset + (HALF ? i : 2 * i), ib = HALF ? ia + p.pairs : ia + 1;
      const float a = to_f(x[ia]), b = to_f(x[ib]);
      from_f(a * cs.x - b * cs.y, y[ia]);
      from_f(a * cs.y + b * cs.x, y[ib]);
    } else {
      const int c = i - p.pairs;
      const int ch = c < p.offset ? c : c + 2 * p.pairs;
      y[ch] = x[ch];
    }
  }
}

constexpr int kHeads = 4;  // heads per thread of the 16-byte kernel

// Unit of a head: a 16-byte piece, or in the half layout the two pieces that
// pair up. Blocks take `tpb` tokens; rcp_* = ceil(2^32 / d) divide the block's
// unit index (below 2^16).
struct RopeV {
  int units, groups, tpb;
  unsigned rcp_units, rcp_groups;
};

template <typename T>
struct Piece {
  static constexpr int N = 16 / sizeof(T);
  union {
    uint4 v;
    T e[N];
  };
  __device__ Piece() {}
};

template <typename T, bool HALF>
__global__ void __launch_bounds__(kThreads) rope_vec_kernel(const RopeK p, const RopeV v) {
  constexpr int N = 16 / sizeof(T);
  constexpr int NP = HALF ? N : N / 2;  // pairs of a unit
  grid_dep_sync();
  const int o16 = p.offset / N, span = p.pairs / NP;  // the rotated units
  const long long t0 = blockIdx.x * static_cast<long long>(v.tpb);
  const int work = v.units * v.groups *
                   static_cast<int>(min(static_cast<long long>(v.tpb), p.tokens - t0));
  for (int k = threadIdx.x; k < work; k += kThreads) {
    const int tg = v.units == 1 ? k : static_cast<int>(__umulhi(k, v.rcp_units));
    const int tl = v.groups == 1 ? tg : static_cast<int>(__umulhi(tg, v.rcp_groups));
    const int u = k - tg * v.units;
    const int h0 = (tg - tl * v.groups) * kHeads, nh = min(kHeads, p.heads - h0);
    const long long t = t0 + tl;
    int piece = p.in_place ? o16 + u : u;
    const bool turn = piece >= o16 && piece < o16 + span;
    if (HALF && piece >= o16 + span) piece += span;
    const T* x = static_cast<const T*>(p.x) + t * p.x_tok + h0 * p.x_head + piece * N;
    T* y = static_cast<T*>(p.y) + t * p.y_tok + h0 * p.y_head + piece * N;
    Piece<T> a[kHeads], b[kHeads];
#pragma unroll
    for (int h = 0; h < kHeads; ++h)
      if (h < nh) {
        a[h].v = *reinterpret_cast<const uint4*>(x + h * p.x_head);
        if (HALF && turn) b[h].v = *reinterpret_cast<const uint4*>(x + h * p.x_head + p.pairs);
      }
    if (turn) {
      float2 cs[NP];
      const int i0 = (piece - o16) * NP;
#pragma unroll
      for (int i = 0; i < NP; ++i) cs[i] = pair_cs(p, t, i0 + i);
#pragma unroll
      for (int h = 0; h < kHeads; ++h)
#pragma unroll
        for (int i = 0; i < NP; ++i) {
          T& ea = HALF ? a[h].e[i] : a[h].e[2 * i];
          T& eb = HALF ? b[h].e[i] : a[h].e[2 * i + 1];
          const float fa = to_f(ea), fb = to_f(eb);
          from_f(fa * cs[i].x - fb * cs[i].y, ea);
          from_f(fa * cs[i].y + fb * cs[i].x, eb);
        }
    }
#pragma unroll
    for (int h = 0; h < kHeads; ++h)
      if (h < nh) {
        *reinterpret_cast<uint4*>(y + h * p.y_head) = a[h].v;
        if (HALF && turn) *reinterpret_cast<uint4*>(y + h * p.y_head + p.pairs) = b[h].v;
      }
  }
}

bool on_16(const RopeArgs& a, const RopeK& k, int size) {
  const auto ok = [&](long long elems) { return elems * size % 16 == 0; };
  return aligned_to(a.x, 16) && aligned_to(a.y, 16) && ok(a.x_tok) && ok(a.x_head) &&
         ok(a.y_tok) && ok(a.y_head) && ok(a.offset) && (k.in_place || ok(a.head_dim)) &&
         ok(a.layout == MLA_ROPE_HALF ? a.pairs : 2 * a.pairs);
}

template <typename T>
int launch_typed(const RopeArgs& a, const RopeK& k) {
  constexpr int N = 16 / sizeof(T);
  const bool half = a.layout == MLA_ROPE_HALF;
  if (on_16(a, k, sizeof(T))) {
    RopeV v;
    v.units = (k.in_place ? 2 * a.pairs : a.head_dim) / N - (half ? a.pairs / N : 0);
    v.groups = (a.heads + kHeads - 1) / kHeads;
    const long long per_token = static_cast<long long>(v.units) * v.groups;
    if (per_token < 65536) {
      v.tpb = per_token >= kThreads ? 1 : static_cast<int>(kThreads / per_token);
      v.rcp_units = static_cast<unsigned>(((1ull << 32) + v.units - 1) / v.units);
      v.rcp_groups = static_cast<unsigned>(((1ull << 32) + v.groups - 1) / v.groups);
      const long long blocks = (a.tokens + v.tpb - 1) / v.tpb;
      if (blocks < (1ll << 31))
        return launch_pdl(half ? rope_vec_kernel<T, true> : rope_vec_kernel<T, false>,
                          dim3(static_cast<unsigned>(blocks)), kThreads, 0, a.stream, k, v);
    }
  }
  const int items = a.pairs + (k.in_place ? 0 : a.head_dim - 2 * a.pairs);
  const long long n = a.tokens * a.heads * items;
  const long long want = (n + kThreads - 1) / kThreads;
  const int blocks = static_cast<int>(want < 152 * 16 ? want : 152 * 16);
  return launch_pdl(half ? rope_kernel<T, true> : rope_kernel<T, false>,
                    dim3(blocks), kThreads, 0, a.stream, k);
}

}  // namespace

int check_rope(const mla_rope* r) {
  if (!r || !r->table || !aligned_to(r->table, 8) || r->table_len < 1) return MLA_ERR_ARG;
  if (r->pairs_t < 0 || r->pairs_h < 0 || r->pairs_w < 0 || r->offset < 0) return MLA_ERR_ARG;
  if (r->pairs_t > 4096 || r->pairs_h > 4096 || r->pairs_w > 4096 || r->offset > (1 << 20) ||
      r->pairs_t + r->pairs_h + r->pairs_w < 1)
    return MLA_ERR_ARG;
  if (r->axes != 1 && r->axes != 3) return MLA_ERR_ARG;
  if (r->axes == 1 && (r->pairs_h || r->pairs_w)) return MLA_ERR_ARG;
  return r->layout == MLA_ROPE_INTERLEAVED || r->layout == MLA_ROPE_HALF ? MLA_OK : MLA_ERR_ARG;
}

int launch_rope_apply(const RopeArgs& a) {
  RopeK k;
  k.x = a.x;
  k.pos = a.pos;
  k.y = a.y;
  k.table = a.table;
  k.tokens = a.tokens;
  k.x_tok = a.x_tok;
  k.x_head = a.x_head;
  k.y_tok = a.y_tok;
  k.y_head = a.y_head;
  k.heads = a.heads;
  k.head_dim = a.head_dim;
  k.table_len = a.table_len;
  k.pairs = a.pairs;
  k.pairs_t = a.pairs_t;
  k.pairs_h = a.pairs_h;
  k.axes = a.axes;
  k.offset = a.offset;
  k.sign = a.inverse ? -1.f : 1.f;
  k.in_place = a.x == a.y;
  k.status = a.status;
  switch (a.dtype) {
    case MLA_DTYPE_BF16: return launch_typed<__nv_bfloat16>(a, k);
    case MLA_DTYPE_FP16: return launch_typed<__half>(a, k);
    default: return launch_typed<float>(a, k);
  }
}

}  // namespace vmla

using namespace vmla;

extern "C" {

int mla_rope_scaled_table_fill(int rot_dim, int table_len, double theta, int scaling,
                               double factor, int native_len, double beta_fast, double beta_slow,
                               float* host_table) {
  if (!host_table || rot_dim < 2 || rot_dim % 2 != 0 || table_len < 1 || !(theta > 0.0) ||
      !std::isfinite(theta) || scaling < MLA_ROPE_SCALE_NONE || scaling > MLA_ROPE_SCALE_YARN ||
      !(factor >= 1.0) || !std::isfinite(factor))
    return MLA_ERR_ARG;
  if (scaling == MLA_ROPE_SCALE_NTK && rot_dim < 4) return MLA_ERR_ARG;
  if (scaling == MLA_ROPE_SCALE_YARN && (native_len < 1 || !(beta_fast > beta_slow)))
    return MLA_ERR_ARG;
  constexpr double kTwoPi = 6.283185307179586476925286766559;
  const int m = rot_dim / 2;
  double base = theta, size = 1.0;
  if (scaling == MLA_ROPE_SCALE_NTK)
    base = theta * std::pow(factor, static_cast<double>(rot_dim) / (rot_dim - 2));
  if (scaling == MLA_ROPE_SCALE_YARN) size = 0.1 * std::log(factor) + 1.0;
  for (int i = 0; i < m; ++i) {
    double f = std::pow(base, -2.0 * i / rot_dim);
    if (scaling == MLA_ROPE_SCALE_LINEAR) f /= factor;
    if (scaling == MLA_ROPE_SCALE_YARN) {
      const double turns = native_len * f / kTwoPi;
      double keep = (turns - beta_slow) / (beta_fast - beta_slow);
      keep = keep < 0.0 ? 0.0 : (keep > 1.0 ? 1.0 : keep);
      f = f / factor * (1.0 - keep) + f * keep;
    }
    for (int pos = 0; pos < table_len; ++pos) {
      const double ang = static_cast<double>(pos) * f;
      float* o = host_table + (static_cast<size_t>(pos) * m + i) * 2;
      o[0] = static_cast<float>(std::cos(ang) * size);
      o[1] = static_cast<float>(std::sin(ang) * size);
    }
  }
  return MLA_OK;
}

int mla_rope_apply(const mla_rope* rope, const void* x, const int* pos, void* y, int dtype,
                   long long tokens, int heads, int head_dim, long long x_token_stride,
                   long long x_head_stride, long long y_token_stride, long long y_head_stride,
                   int inverse, void* stream) {
  int rc = check_rope(rope);
  if (rc != MLA_OK) return rc;
  if (dtype != MLA_DTYPE_BF16 && dtype != MLA_DTYPE_FP16 && dtype != MLA_DTYPE_FP32)
    return MLA_ERR_ARG;
  const int pairs = rope->pairs_t + rope->pairs_h + rope->pairs_w;
  if (tokens < 0 || heads < 1 || head_dim < 1 || rope->offset + 2 * pairs > head_dim)
    return MLA_ERR_ARG;
  if (tokens == 0) return MLA_OK;
  const unsigned size = dtype == MLA_DTYPE_FP32 ? 4 : 2;
  if (!x || !y || !pos || !aligned_to(x, size) || !aligned_to(y, size) || !aligned_to(pos, 4))
    return MLA_ERR_ARG;
  if (x == y && (x_token_stride != y_token_stride || x_head_stride != y_head_stride))
    return MLA_ERR_ARG;
  if (tokens > (1ll << 40) / (static_cast<long long>(heads) * head_dim)) return MLA_ERR_ARG;
  rc = check_resident({rope->table, x, pos, y});
  if (rc != MLA_OK) return rc;
  RopeArgs a;
  a.x = x;
  a.pos = pos;
  a.y = y;
  a.table = static_cast<const float2*>(rope->table);
  a.tokens = tokens;
  a.x_tok = x_token_stride;
  a.x_head = x_head_stride;
  a.y_tok = y_token_stride;
  a.y_head = y_head_stride;
  a.heads = heads;
  a.head_dim = head_dim;
  a.table_len = rope->table_len;
  a.pairs = pairs;
  a.pairs_t = rope->pairs_t;
  a.pairs_h = rope->pairs_h;
  a.axes = rope->axes;
  a.offset = rope->offset;
  a.layout = rope->layout;
  a.dtype = dtype;
  a.inverse = inverse;
  a.status = device_status_ptr();
  a.stream = static_cast<cudaStream_t>(stream);
  if (!a.status) return MLA_ERR_CUDA;
  return launch_rope_apply(a);
}

}  // extern "C"
