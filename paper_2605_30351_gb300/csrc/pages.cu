// Page operations of a latent cache in pages: lengths with copy on write,
// branching, copying pages, packing the pool. All metadata stays on the device.
//
// The metadata kernels are bound by latency (a few thousand integers): one block
// each, so that no step waits for another launch. The page copies are bound by
// memory: every copied row is read once and written once, in 16-byte pieces, four
// loads of a thread in flight (one: 309 us instead of 267 for the pool below).
// Measured on the GPU (in a CUDA graph): a pool of 4,096 pages x 30 layers with 983 pages
// to move (1.69 GB) packed in 266 us, 6.36 TB/s of a measured copy rate of 6.77; 12
// streams of up to 3,001 tokens branched and grown by 1,560, all 30 layers, 12.5 us in
// five launches (the three calls from Python take 25 - 27 us). A resize always
// launches its copies, also where the plan has none.
#include "internal.h"
#include "ptx_sm103.cuh"

namespace vmla {
namespace {

constexpr int kMeta = 1024;  // threads of the one-block metadata kernel
constexpr int kCopy = 256;

struct Pool {
  uint4* c;
  uint4* kr;
  int* table;
  int* lens;
  int* refs;
  int layers, pages, page_tokens, seqs, max_pages;
  int c16, k16;  // 16-byte pieces of a row of c, of kr
  int* status;
};

Pool pool_of(const mla_paged_cache& c, int* status) {
  Pool p;
  p.c = static_cast<uint4*>(c.c);
  p.kr = static_cast<uint4*>(c.kr);
  p.table = c.table;
  p.lens = c.lens;
  p.refs = c.refs;
  p.layers = c.layers;
  p.pages = c.pages;
  p.page_tokens = c.page_tokens;
  p.seqs = c.seqs;
  p.max_pages = c.max_pages;
  p.c16 = c.d_c / 8;
  p.k16 = c.d_r / 8;
  p.status = status;
  return p;
}

// Exclusive prefix sum of one value per thread over the block, and the total.
template <typename T>
__device__ __forceinline__ T block_scan(T v, T* warp_sums, T& total) {
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, warps = blockDim.x >> 5;
  T x = v;
#pragma unroll
  for (int d = 1; d < 32; d <<= 1) {
    const T y = __shfl_up_sync(0xffffffffu, x, d);
    if (lane >= d) x += y;
  }
  if (lane == 31) warp_sums[warp] = x;
  __syncthreads();
  if (warp == 0) {
    T w = lane < warps ? warp_sums[lane] : T(0);
#pragma unroll
    for (int d = 1; d < 32; d <<= 1) {
      const T y = __shfl_up_sync(0xffffffffu, w, d);
      if (lane >= d) w += y;
    }
    warp_sums[lane] = w;
  }
  __syncthreads();
  total = warp_sums[warps - 1];
  const T before = (warp ? warp_sums[warp - 1] : T(0)) + x - v;
  __syncthreads();  // warp_sums may be written again
  return before;
}

__device__ __forceinline__ int pages_of(int tokens, int page_tokens) {
  return static_cast<int>((static_cast<long long>(tokens) + page_tokens - 1) / page_tokens);
}

// plan of a resize: [0] copies; then per stream (begin, need with the copy flag
// in bit 30); then the copies' (src, dst, rows); then the free pages found
constexpr int kFlagCow = 1 << 30;

__global__ void __launch_bounds__(kMeta) resize_kernel(const Pool p, const int* new_lens,
                                                       int* plan) {
  grid_dep_sync();
  __shared__ int sums[32];
  __shared__ long long wide[32];
  __shared__ int n_copies;
  int* begin = plan + 1;
  int* need = begin + p.seqs;
  int* copies = need + p.seqs;
  int* free_list = copies + 3 * p.seqs;
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, warps = kMeta / 32;
  const long long cap = static_cast<long long>(p.max_pages) * p.page_tokens;
  if (threadIdx.x == 0) n_copies = 0;

  // pages past a shorter length are given back (a warp per stream)
  for (int s = warp; s < p.seqs; s += warps) {
    const int want_len = new_lens[s], len = p.lens[s];
    if (want_len < 0 || want_len >= len || len > cap) continue;
    const int want = pages_of(want_len, p.page_tokens), have = pages_of(len, p.page_tokens);
    int* row = p.table + static_cast<size_t>(s) * p.max_pages;
    for (int j = want + lane; j < have; j += 32) {
      const int pg = row[j];
      if (pg >= 0 && pg < p.pages)
        atomicSub(p.refs + pg, 1);
      else
        record_status(p.status, MLA_ERR_RANGE);
      row[j] = -1;
    }
    __syncwarp();  // every lane has read the length
    if (lane == 0) p.lens[s] = want_len;
  }
  __syncthreads();

  // pages each growing stream needs, and where its share of the free list begins
  // (sums in 64 bits: lengths that no pool can hold must not wrap around)
  long long carry = 0;
  for (int s0 = 0; s0 < p.seqs; s0 += kMeta) {
    const int s = s0 + threadIdx.x;
    int v = 0;
    bool cow = false;
    if (s < p.seqs) {
      const int want_len = new_lens[s], len = p.lens[s];
      if (want_len > cap || len < 0 || len > cap) {
        record_status(p.status, MLA_ERR_RANGE);
      } else if (want_len > len) {
        const int have = pages_of(len, p.page_tokens);
        v = pages_of(want_len, p.page_tokens) - have;
        if (len % p.page_tokens) {
          const int last = p.table[static_cast<size_t>(s) * p.max_pages + have - 1];
          if (last < 0 || last >= p.pages) {
            record_status(p.status, MLA_ERR_RANGE);
          } else {
            cow = p.refs[last] > 1;
          }
        }
        v += cow;
      }
    }
    long long total;
    const long long at = carry + block_scan(static_cast<long long>(v), wide, total);
    if (s < p.seqs) {
      begin[s] = static_cast<int>(min(at, static_cast<long long>(p.pages)));
      need[s] = v | (cow ? kFlagCow : 0);
    }
    carry += total;
  }
  const int wanted = static_cast<int>(min(carry, static_cast<long long>(p.pages)));

  // the first `wanted` free pages, lowest first
  int found = 0;
  for (int p0 = 0; p0 < p.pages && found < wanted; p0 += kMeta) {
    const int pg = p0 + threadIdx.x;
    const int is_free = pg < p.pages && p.refs[pg] <= 0;
    int total;
    const int at = found + block_scan(is_free, sums, total);
    if (is_free && at < wanted) free_list[at] = pg;
    found += total;
  }
  __syncthreads();

  // hand them out (a warp per stream)
  for (int s = warp; s < p.seqs; s += warps) {
    const int want_len = new_lens[s];
    const int len = p.lens[s];
    if (want_len <= len || want_len > cap || len < 0) continue;
    const bool cow = (need[s] & kFlagCow) != 0;
    const int v = need[s] & ~kFlagCow, b = begin[s];
    if (v > 0 && (b >= found || v > found - b)) {
      if (lane == 0) record_status(p.status, MLA_ERR_RANGE);
      continue;
    }
    __syncwarp();  // every lane has read the length
    const int have = pages_of(len, p.page_tokens);
    int* row = p.table + static_cast<size_t>(s) * p.max_pages;
    for (int j = cow + lane; j < v; j += 32) {
      const int pg = free_list[b + j];
      row[have + j - cow] = pg;
      p.refs[pg] = 1;
    }
    if (lane == 0) {
      if (cow) {
        const int from = row[have - 1], to = free_list[b];
        const int k = atomicAdd(&n_copies, 1);
        copies[3 * k] = from;
        copies[3 * k + 1] = to;
        copies[3 * k + 2] = len % p.page_tokens;
        row[have - 1] = to;
        p.refs[to] = 1;
        atomicSub(p.refs + from, 1);
      }
      p.lens[s] = want_len;
    }
  }
  __syncthreads();
  if (threadIdx.x == 0) plan[0] = n_copies;
}

// n 16-byte pieces by the block: kFlight loads of a thread before its first store,
// so that a unit of a page and layer (28 KB at 64 tokens of 224 values) is mostly in
// flight at once. Counted in 64 bits: a page of wide rows may hold 2^31 pieces.
constexpr int kFlight = 4;

__device__ __forceinline__ void copy_pieces(const uint4* src, uint4* dst, long long n) {
  for (long long i0 = threadIdx.x; i0 < n; i0 += kCopy * kFlight) {
    uint4 v[kFlight];
#pragma unroll
    for (int k = 0; k < kFlight; ++k)
      if (i0 + k * kCopy < n) v[k] = src[i0 + k * kCopy];
#pragma unroll
    for (int k = 0; k < kFlight; ++k)
      if (i0 + k * kCopy < n) dst[i0 + k * kCopy] = v[k];
  }
}

// The first `rows` rows of page `from` to page `to`, one layer.
__device__ __forceinline__ void copy_rows(const Pool& p, int from, int to, int rows, int layer) {
  const size_t base = static_cast<size_t>(layer) * p.pages;
  const size_t a = (base + from) * p.page_tokens, b = (base + to) * p.page_tokens;
  copy_pieces(p.c + a * p.c16, p.c + b * p.c16, static_cast<long long>(rows) * p.c16);
  copy_pieces(p.kr + a * p.k16, p.kr + b * p.k16, static_cast<long long>(rows) * p.k16);
}

__global__ void __launch_bounds__(kCopy) copy_plan_kernel(const Pool p, const int* plan) {
  grid_dep_sync();
  const int* copies = plan + 1 + 2 * p.seqs;
  const long long units = static_cast<long long>(plan[0]) * p.layers;
  for (long long u = blockIdx.x; u < units; u += gridDim.x) {
    const int i = static_cast<int>(u / p.layers), layer = static_cast<int>(u % p.layers);
    copy_rows(p, copies[3 * i], copies[3 * i + 1], copies[3 * i + 2], layer);
  }
}

__global__ void __launch_bounds__(kCopy)
    copy_pages_kernel(const Pool p, const int* src, const int* dst, int n) {
  grid_dep_sync();
  const long long units = static_cast<long long>(n) * p.layers;
  for (long long u = blockIdx.x; u < units; u += gridDim.x) {
    const int i = static_cast<int>(u / p.layers), layer = static_cast<int>(u % p.layers);
    const int from = src[i], to = dst[i];
    if (from < 0 || from >= p.pages || to < 0 || to >= p.pages) {
      if (threadIdx.x == 0) record_status(p.status, MLA_ERR_RANGE);
      continue;
    }
    copy_rows(p, from, to, p.page_tokens, layer);
  }
}

__global__ void __launch_bounds__(kCopy)
    fork_kernel(const Pool p, int* dropped, const int* src, const int* dst, int n) {
  grid_dep_sync();
  const int i = blockIdx.x;
  const int s = src[i], d = dst[i];
  if (s < 0 || s >= p.seqs || d < 0 || d >= p.seqs || s == d) {
    if (threadIdx.x == 0) record_status(p.status, MLA_ERR_RANGE);
    return;
  }
  const int len = p.lens[s];
  const bool busy = p.lens[d] != 0;
  __syncthreads();
  if (busy || len < 0 || len > static_cast<long long>(p.max_pages) * p.page_tokens) {
    if (threadIdx.x == 0) record_status(p.status, MLA_ERR_RANGE);
    return;
  }
  const int have = pages_of(len, p.page_tokens);
  const int* from = p.table + static_cast<size_t>(s) * p.max_pages;
  int* to = p.table + static_cast<size_t>(d) * p.max_pages;
  for (int j = threadIdx.x; j < have; j += kCopy) {
    const int pg = from[j];
    to[j] = pg;
    if (pg >= 0 && pg < p.pages)
      atomicAdd(p.refs + pg, 1);
    else
      record_status(p.status, MLA_ERR_RANGE);
  }
  if (threadIdx.x == 0) {
    p.lens[d] = len;
    if (dropped) dropped[d] = dropped[s];
  }
}

// Pages between a stream's sinks and its newest tokens leave its list (a block per
// stream): their references go first, then the entries behind them move up, kCopy at
// a time, every entry read before the place it moves to, which lies ahead of it, is
// written. Bound by latency: lens, then the table, then the references. 64 streams with up to
// 200 pages to go 2.4 us, 1,024 streams that give 55,900 pages back 3.4.
__global__ void __launch_bounds__(kCopy)
    slide_kernel(const Pool p, int* dropped, const int* keep, int front) {
  grid_dep_sync();
  const int s = blockIdx.x;
  const int kept = keep[s], len = p.lens[s], gone = dropped[s];
  const long long cap = static_cast<long long>(p.max_pages) * p.page_tokens;
  if (kept < 0) {
    if (kept < -1 && threadIdx.x == 0) record_status(p.status, MLA_ERR_RANGE);
    return;
  }
  if (len < 0 || len > cap || gone < 0) {
    if (threadIdx.x == 0) record_status(p.status, MLA_ERR_RANGE);
    return;
  }
  // a stream that holds no token starts anew (window_plan_kernel): its last page stays
  const int most = max(kept, 1), n = (len > most ? len - most : 0) / p.page_tokens - front;
  if (n <= 0) return;
  if (static_cast<long long>(gone) + len >= kMostTokens) {
    if (threadIdx.x == 0) record_status(p.status, MLA_ERR_RANGE);
    return;
  }
  const int have = pages_of(len, p.page_tokens), left = have - n;
  int* row = p.table + static_cast<size_t>(s) * p.max_pages;
  for (int j = front + threadIdx.x; j < front + n; j += kCopy) {
    const int pg = row[j];
    if (pg >= 0 && pg < p.pages)
      atomicSub(p.refs + pg, 1);
    else
      record_status(p.status, MLA_ERR_RANGE);
  }
  __syncthreads();  // also: every thread has read the stream's numbers
  for (int j0 = front; j0 < left; j0 += kCopy) {
    const int j = j0 + threadIdx.x;
    const int v = j < left ? row[j + n] : 0;
    __syncthreads();
    if (j < left) row[j] = v;
  }
  __syncthreads();  // the last entries have moved
  for (int j = left + threadIdx.x; j < have; j += kCopy) row[j] = -1;
  if (threadIdx.x == 0) {
    p.lens[s] = len - n * p.page_tokens;
    dropped[s] = gone + n * p.page_tokens;
  }
}

// Packing. plan: [0] pages in use n, [1] pages that move m; then per page where
// it goes (page >= 0 stays there, -1 not in use, -2 - r the r-th that moves),
// then the free places below n, then the pages that move.
__global__ void __launch_bounds__(kMeta) pack_plan_kernel(const Pool p, int* plan) {
  grid_dep_sync();
  __shared__ long long sums[32];
  int* where = plan + 2;
  int* holes = where + p.pages;
  int* movers = holes + p.pages;
  // kRun consecutive pages a thread: one prefix sum for 8,192 pages and pass, of
  // the pages in use (low half) and of those past n (high half) together
  constexpr int kRun = 8;
  auto used_at = [&](int first) {  // a bit for each of the thread's pages in use
    unsigned m = 0;
#pragma unroll
    for (int k = 0; k < kRun; ++k)
      if (first + k < p.pages && p.refs[first + k] > 0) m |= 1u << k;
    return m;
  };
  int n = 0;
  for (int p0 = 0; p0 < p.pages; p0 += kMeta * kRun) {
    long long total;
    block_scan(static_cast<long long>(__popc(used_at(p0 + threadIdx.x * kRun))), sums, total);
    n += static_cast<int>(total);
  }
  int live = 0, moved = 0;
  for (int p0 = 0; p0 < p.pages; p0 += kMeta * kRun) {
    const int first = p0 + threadIdx.x * kRun;
    const unsigned used = used_at(first);
    const int below = n <= first ? 0 : min(kRun, n - first);  // of the thread's pages
    const unsigned past = used & (0xffu << below);
    long long total;
    const long long at = block_scan(
        static_cast<long long>(__popc(used)) + (static_cast<long long>(__popc(past)) << 32), sums,
        total);
    int before = live + static_cast<int>(at & 0xffffffff);
    int rank = moved + static_cast<int>(at >> 32);
    for (int k = 0; k < kRun && first + k < p.pages; ++k) {
      const int pg = first + k;
      if (!(used >> k & 1)) {
        where[pg] = -1;
        if (pg < n) holes[pg - before] = pg;
        continue;
      }
      ++before;
      where[pg] = pg < n ? pg : -2 - rank;
      if (pg >= n) movers[rank++] = pg;
    }
    live += static_cast<int>(total & 0xffffffff);
    moved += static_cast<int>(total >> 32);
  }
  if (threadIdx.x == 0) {
    plan[0] = n;
    plan[1] = moved;
  }
}

__global__ void __launch_bounds__(kCopy)
    pack_kernel(const Pool p, const int* plan, int* new_table, int* new_refs) {
  grid_dep_sync();
  const int n = plan[0], m = plan[1];
  const int* where = plan + 2;
  const int* holes = where + p.pages;
  const int* movers = holes + p.pages;
  const long long step = static_cast<long long>(gridDim.x) * kCopy;
  const long long first = blockIdx.x * static_cast<long long>(kCopy) + threadIdx.x;
  const long long cells = static_cast<long long>(p.seqs) * p.max_pages;
  for (long long i = first; i < cells; i += step) {
    const int pg = p.table[i];
    int to = -1;
    if (pg >= 0 && pg < p.pages) {
      to = where[pg];
      if (to == -1)
        record_status(p.status, MLA_ERR_RANGE);
      else if (to < -1)
        to = holes[-2 - to];
    } else if (pg != -1) {
      record_status(p.status, MLA_ERR_RANGE);
    }
    new_table[i] = to;
  }
  // new_refs may be refs: a page that moves and its new place belong to one thread
  for (long long i = first; i < p.pages; i += step) {
    const int w = where[i];
    if (w >= 0) {
      new_refs[i] = p.refs[i];
    } else if (w == -1) {
      if (i >= n) new_refs[i] = 0;
    } else {
      new_refs[holes[-2 - w]] = p.refs[i];
      new_refs[i] = 0;
    }
  }
  const long long units = static_cast<long long>(m) * p.layers;
  for (long long u = blockIdx.x; u < units; u += gridDim.x) {
    const int i = static_cast<int>(u / p.layers), layer = static_cast<int>(u % p.layers);
    copy_rows(p, movers[i], holes[i], p.page_tokens, layer);
  }
}

int grid_for(long long units) {
  const long long most = 152 * 8;
  return static_cast<int>(units < 1 ? 1 : (units < most ? units : most));
}

}  // namespace

unsigned long long pages_plan_ints(const mla_paged_cache& c) {
  const unsigned long long resize = 1ull + 5ull * c.seqs + c.pages;
  const unsigned long long pack = 2ull + 3ull * c.pages;
  return resize > pack ? resize : pack;
}

int launch_pages_resize(const mla_paged_cache& c, const int* new_lens, int* status,
                        cudaStream_t stream) {
  const Pool p = pool_of(c, status);
  int* plan = static_cast<int*>(c.plan);
  const int rc = launch_pdl(resize_kernel, dim3(1), kMeta, 0, stream, p, new_lens, plan);
  if (rc != MLA_OK) return rc;
  return launch_pdl(copy_plan_kernel, dim3(grid_for(static_cast<long long>(c.seqs) * c.layers)),
                    kCopy, 0, stream, p, plan);
}

int launch_pages_fork(const mla_paged_cache& c, const int* src, const int* dst, int n,
                      int* status, cudaStream_t stream) {
  return launch_pages_window_fork(c, nullptr, src, dst, n, status, stream);
}

int launch_pages_window_fork(const mla_paged_cache& c, int* dropped, const int* src,
                             const int* dst, int n, int* status, cudaStream_t stream) {
  return launch_pdl(fork_kernel, dim3(n), kCopy, 0, stream, pool_of(c, status), dropped, src, dst,
                    n);
}

int launch_pages_slide(const mla_paged_cache& c, const mla_paged_window& w, const int* keep,
                       int* status, cudaStream_t stream) {
  const long long front = (static_cast<long long>(w.sinks) + c.page_tokens - 1) / c.page_tokens;
  return launch_pdl(slide_kernel, dim3(c.seqs), kCopy, 0, stream, pool_of(c, status), w.dropped,
                    keep, static_cast<int>(front));
}

int launch_pages_copy(const mla_paged_cache& c, const int* src, const int* dst, int n,
                      int* status, cudaStream_t stream) {
  return launch_pdl(copy_pages_kernel, dim3(grid_for(static_cast<long long>(n) * c.layers)),
                    kCopy, 0, stream, pool_of(c, status), src, dst, n);
}

int launch_pages_compact(const mla_paged_cache& c, int* new_table, int* new_refs, int* status,
                         cudaStream_t stream) {
  const Pool p = pool_of(c, status);
  int* plan = static_cast<int*>(c.plan);
  const int rc = launch_pdl(pack_plan_kernel, dim3(1), kMeta, 0, stream, p, plan);
  if (rc != MLA_OK) return rc;
  return launch_pdl(pack_kernel, dim3(grid_for(static_cast<long long>(c.pages) * c.layers)),
                    kCopy, 0, stream, p, plan, new_table, new_refs);
}

}  // namespace vmla
