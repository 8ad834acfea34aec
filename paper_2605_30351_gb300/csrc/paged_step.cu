// The metadata of a step of many streams, made on the GPU from their lengths: the places
// of the step's rows and the lengths to grow to, then the new tokens' coordinates and
// rows of the pool. A stream's index of a token is its place among the held ones plus
// what was given back (App. D.4); the sinks' coordinates are those of App. D.5.
//
// Both are bound by latency (a launch, then one or two dependent loads). Measured on the GPU:
// the plan of 64 streams 1.5 us, of 65,536 4.4; positions and rows of 64 tokens 2.6 us, of
// 30,900 2.3. A call from Python takes 6 - 7.5 us: two thirds of it the binding and the launch.
#include "internal.h"
#include "paged_attn.cuh"
#include "ptx_sm103.cuh"

namespace vmla {
namespace {

constexpr int kPlan = 1024;
constexpr int kPos = 256;

// A thread per stream; each block adds up the counts before its own by itself, so that no
// block waits for another (65,536 streams: 64 blocks read 8 MB of counts from L2 in all; one
// block that walks all streams takes 117 us longer). Sums in 64 bits.
__global__ void __launch_bounds__(kPlan)
    window_plan_kernel(const int* lens, int* dropped, const int* n_new, int* q_start,
                       int* new_lens, int seqs, int* status) {
  constexpr int kWarps = kPlan / 32, kFlight = 8;
  __shared__ long long sums[kWarps], before[kWarps];
  grid_dep_sync();
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  constexpr long long kTop = 0x7fffffff;
  const int s0 = blockIdx.x * kPlan, s = s0 + threadIdx.x;
  int n = 0, len = 0;
  if (s < seqs) {
    n = n_new[s];
    len = lens[s];
  }
  long long pre = 0;
  for (int i = threadIdx.x; i < s0; i += kPlan * kFlight) {
    int v[kFlight];
#pragma unroll
    for (int k = 0; k < kFlight; ++k) v[k] = i + k * kPlan < s0 ? n_new[i + k * kPlan] : 0;
#pragma unroll
    for (int k = 0; k < kFlight; ++k) pre += max(v[k], 0);
  }
  if (s < seqs) {
    if (n < 0 || (n > 0 && len > kTop - n)) record_status(status, MLA_ERR_RANGE);
    n = max(n, 0);
    if (len == 0 && dropped) dropped[s] = 0;
    new_lens[s] = n > 0 ? static_cast<int>(min(static_cast<long long>(len) + n, kTop)) : -1;
  }
  long long x = n;
#pragma unroll
  for (int d = 1; d < 32; d <<= 1) {
    const long long y = __shfl_up_sync(0xffffffffu, x, d);
    if (lane >= d) x += y;
    pre += __shfl_xor_sync(0xffffffffu, pre, d);
  }
  if (lane == 31) {
    sums[warp] = x;
    before[warp] = pre;
  }
  __syncthreads();
  // every warp adds up the warps before its own, and what the blocks before hold
  long long y = before[lane] + (lane < warp ? sums[lane] : 0);
#pragma unroll
  for (int d = 1; d < 32; d <<= 1) y += __shfl_xor_sync(0xffffffffu, y, d);
  if (s == 0) q_start[0] = 0;
  if (s < seqs) {
    if (y + x > kTop) record_status(status, MLA_ERR_RANGE);
    q_start[s + 1] = static_cast<int>(min(y + x, kTop));
  }
}

struct PositionsK {
  const int* q_start;
  const int* table;
  const int* lens;
  const int* dropped;
  int* pos;
  int* pos_sink;
  int* rows;
  int total, seqs, pages, page_tokens, max_pages, window, sinks, front, block, axes;
  int frame, width;
  Div by_page, by_mask, by_frame, by_width;
  int* status;
};

// A thread per token. The block's first and last token bound the streams that its
// tokens may be of; each thread searches between them.
__global__ void __launch_bounds__(kPos) window_positions_kernel(const PositionsK p) {
  __shared__ int bounds[2];
  grid_dep_sync();
  if (blockIdx.x == 0) check_q_start(p.q_start, p.seqs, p.total, p.status);
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const long long first = static_cast<long long>(blockIdx.x) * kPos;
  if (warp < 2) {
    const long long t = min(first + (warp ? kPos - 1 : 0), static_cast<long long>(p.total) - 1);
    const int s = stream_of(p.q_start, p.seqs, static_cast<int>(t), lane);
    if (lane == 0) bounds[warp] = s;
  }
  __syncthreads();
  const long long at = first + threadIdx.x;
  if (at >= p.total) return;
  const int t = static_cast<int>(at);
  int lo = bounds[0], hi = max(bounds[0], bounds[1]);
  while (lo < hi) {
    const int mid = (lo + hi + 1) / 2;
    if (p.q_start[mid] <= t)
      lo = mid;
    else
      hi = mid - 1;
  }
  const int q0 = p.q_start[lo], q1 = p.q_start[lo + 1];
  if (t < q0 || t >= q1 || q1 > p.total) return;  // check_q_start records it
  const int len = p.lens[lo], gone = p.dropped ? p.dropped[lo] : 0;
  int g = 0, hidden = 0, row = -1;
  const long long place = static_cast<long long>(len) - (q1 - q0) + (t - q0);
  if (len < 0 || gone < 0 || static_cast<long long>(len) + gone >= kMostTokens ||
      (gone > 0 && static_cast<long long>(len) - (q1 - q0) < p.front)) {
    // no stream, or new tokens among the sinks' pages of one that gave tokens back: attention
    // refuses the same (stream_held)
    record_status(p.status, MLA_ERR_RANGE);
  } else if (place >= 0) {
    const int j = p.by_page(static_cast<int>(place));
    if (j < p.max_pages) {
      const int page = p.table[static_cast<size_t>(lo) * p.max_pages + j];
      if (page >= 0 && page < p.pages)
        row = page * p.page_tokens + static_cast<int>(place - static_cast<long long>(j) * p.page_tokens);
    }
    g = static_cast<int>(place) + gone;
    long long end = len + gone;
    if (p.block > 0) end = min(end, static_cast<long long>(p.by_mask(g) + 1) * p.block);
    hidden = static_cast<int>(max(0ll, end - p.window - p.sinks));
  }
  if (row < 0) record_status(p.status, MLA_ERR_RANGE);
  if (p.rows) p.rows[t] = row;
  const int f = p.by_frame(g), f_sink = f - p.by_frame(hidden);
  if (p.axes == 1) {
    p.pos[t] = f;
    if (p.pos_sink) p.pos_sink[t] = f_sink;
    return;
  }
  const int in_frame = g - f * p.frame, h = p.by_width(in_frame), w = in_frame - h * p.width;
  int* y = p.pos + 3ll * t;
  y[0] = f;
  y[1] = h;
  y[2] = w;
  if (p.pos_sink) {
    int* z = p.pos_sink + 3ll * t;
    z[0] = f_sink;
    z[1] = h;
    z[2] = w;
  }
}

}  // namespace

int launch_paged_window_plan(const mla_paged_cache& c, int* dropped, const int* n_new,
                             int* q_start, int* new_lens, int* status, cudaStream_t stream) {
  return launch_pdl(window_plan_kernel, dim3((c.seqs - 1) / kPlan + 1), kPlan, 0, stream, c.lens, dropped, n_new,
                    q_start, new_lens, c.seqs, status);
}

int launch_paged_positions(const PagedPositionsArgs& a) {
  PositionsK k;
  k.q_start = a.q_start;
  k.table = a.table;
  k.lens = a.lens;
  k.dropped = a.dropped;
  k.pos = a.pos;
  k.pos_sink = a.pos_sink;
  k.rows = a.rows;
  k.total = a.total;
  k.seqs = a.seqs;
  k.pages = a.pages;
  k.page_tokens = a.page_tokens;
  k.max_pages = a.max_pages;
  k.window = a.window;
  k.sinks = a.sinks;
  k.front = sink_places(a.sinks, a.page_tokens);
  k.block = a.causal_block;
  k.axes = a.axes;
  k.frame = a.tokens_per_frame;
  k.width = a.frame_width;
  k.by_page = div_by(k.page_tokens);
  k.by_mask = div_by(k.block > 0 ? k.block : 1);
  k.by_frame = div_by(k.frame);
  k.by_width = div_by(k.width);
  k.status = a.status;
  const int blocks = (a.total - 1) / kPos + 1;
  return launch_pdl(window_positions_kernel, dim3(blocks), kPos, 0, a.stream, k);
}

}  // namespace vmla
