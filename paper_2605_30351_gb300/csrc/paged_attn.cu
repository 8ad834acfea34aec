// Attention of ragged streams' newest tokens over a paged latent cache: the choice of a
// kernel, and the join of partial rows. The kernel itself is paged_attn_kernel.cuh.
#include "paged_attn_kernel.cuh"

namespace vmla {
namespace {

constexpr int kJoinThreads = 512;
constexpr int kJoinGrid = kMaxCtas;
constexpr int kJoinCols = 16;  // columns of a warp's join item of 32 rows

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

template <int DC>
int launch_join_pairs(const PagedK& k, int ctas, int cl, const PagedAttnArgs& a) {
  return cl == 2 ? launch_join<DC, DC, 2>(k, ctas, a) : launch_join<DC, DC, 1>(k, ctas, a);
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

int launch_paged_join(const PagedK& k, int ctas, int cl, const PagedAttnArgs& a) {
  switch (a.d_c) {
    case 64: return launch_join_pairs<64>(k, ctas, cl, a);
    case 128: return launch_join_pairs<128>(k, ctas, cl, a);
    case 192: return launch_join_pairs<192>(k, ctas, cl, a);
    case 256: return launch_join_pairs<256>(k, ctas, cl, a);
    case 512: return launch_join<512, 256, 2>(k, ctas, a);
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
  return a.d_r == 32 ? pick_dc<32, false>(a) : pick_dc<64, false>(a);
}

}  // namespace vmla
