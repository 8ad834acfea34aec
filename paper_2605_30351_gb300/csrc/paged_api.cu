// C ABI of the paged latent cache: argument checks and dispatch. See
// include/videomla.h.
#include <cmath>
#include <utility>

#include "internal.h"
#include "ptx_sm103.cuh"

namespace vmla {
namespace {

int check_sizes(const mla_paged_cache* c) {
  if (!c) return MLA_ERR_ARG;
  if (c->layers < 1 || c->pages < 1 || c->page_tokens < 8 || c->seqs < 1 || c->seqs > 65536 ||
      c->max_pages < 1 || c->d_c < 8 || c->d_r < 8 || c->d_c % 8 != 0 || c->d_r % 8 != 0)
    return MLA_ERR_ARG;
  constexpr long long kMost = (1ll << 31) - (1 << 16);
  if (static_cast<long long>(c->pages) * c->page_tokens >= kMost ||
      static_cast<long long>(c->max_pages) * c->page_tokens >= kMost || c->d_c > 65536 ||
      c->d_r > 65536)
    return MLA_ERR_ARG;
  return MLA_OK;
}

// The cache's own buffers are there and aligned, for an operation that needs the plan or not.
int check_buffers(const mla_paged_cache* c, bool plan) {
  const int rc = check_sizes(c);
  if (rc != MLA_OK) return rc;
  if (!c->c || !c->kr || !c->table || !c->lens || !c->refs || (plan && !c->plan))
    return MLA_ERR_ARG;
  if (!aligned_to(c->c, 16) || !aligned_to(c->kr, 16) || !aligned_to(c->table, 16) ||
      !aligned_to(c->lens, 16) || !aligned_to(c->refs, 16) || !aligned_to(c->plan, 16))
    return MLA_ERR_ARG;
  return MLA_OK;
}

// They are this GPU's memory too.
int check_cache(const mla_paged_cache* c, bool plan) {
  const int rc = check_buffers(c, plan);
  if (rc != MLA_OK) return rc;
  return check_resident({c->c, c->kr, c->table, c->lens, c->refs, plan ? c->plan : nullptr});
}

// The window's own rules; dropped may be missing unless the call writes it.
int check_window(const mla_paged_window* w, bool dropped) {
  if (!w || w->window < 1 || w->sinks < 0 || (dropped && !w->dropped) ||
      !aligned_to(w->dropped, 4))
    return MLA_ERR_ARG;
  return MLA_OK;
}

long long table_ints(const mla_paged_cache* c) {
  return static_cast<long long>(c->seqs) * c->max_pages;
}

// Whether two of the arrays (address, ints) share memory.
bool overlap(std::initializer_list<std::pair<const int*, long long>> arrays) {
  for (const auto& a : arrays)
    for (const auto& b : arrays)
      if (&a < &b && a.first && b.first && a.second > 0 && b.second > 0 &&
          a.first < b.first + b.second && b.first < a.first + a.second)
        return true;
  return false;
}

// What both attention calls check, and the arguments without the window's.
int attention_args(const mla_paged_cache* cache, int layer, const void* q_c, const void* q_r,
                   int total, int heads, const int* q_start, int head_dim, int causal_block,
                   void* workspace, unsigned long long workspace_bytes, void* o, void* stream,
                   PagedAttnArgs& a) {
  int rc = check_sizes(cache);
  if (rc != MLA_OK) return rc;
  if (layer < 0 || layer >= cache->layers || total < 0 || heads < 1 || head_dim < 1 ||
      causal_block < 0 || static_cast<long long>(total) * heads > (1ll << 30))
    return MLA_ERR_ARG;
  const unsigned long long need = paged_attention_workspace(cache->d_c, cache->d_r);
  if (need == 0) return MLA_ERR_UNSUPPORTED;
  a.total = total;
  if (total == 0) return check_cache(cache, false);
  if (!q_c || !q_r || !q_start || !workspace || !o || !aligned_to(q_c, 16) ||
      !aligned_to(q_r, 16) || !aligned_to(q_start, 4) || !aligned_to(workspace, 16) ||
      !aligned_to(o, 16) || workspace_bytes < need)
    return MLA_ERR_ARG;
  rc = check_cache(cache, false);
  if (rc == MLA_OK) rc = check_resident({q_c, q_r, q_start, workspace, o});
  if (rc != MLA_OK) return rc;
  const size_t rows = static_cast<size_t>(cache->pages) * cache->page_tokens * layer;
  a.q_c = q_c;
  a.q_r = q_r;
  a.q_start = q_start;
  a.c = static_cast<char*>(cache->c) + rows * cache->d_c * 2;
  a.kr = static_cast<char*>(cache->kr) + rows * cache->d_r * 2;
  a.table = cache->table;
  a.lens = cache->lens;
  a.workspace = workspace;
  a.o = o;
  a.heads = heads;
  a.seqs = cache->seqs;
  a.pages = cache->pages;
  a.page_tokens = cache->page_tokens;
  a.max_pages = cache->max_pages;
  a.d_c = cache->d_c;
  a.d_r = cache->d_r;
  a.causal_block = causal_block;
  a.scale_log2 =
      static_cast<float>(1.4426950408889634 / std::sqrt(static_cast<double>(head_dim)));
  a.status = device_status_ptr();
  a.stream = static_cast<cudaStream_t>(stream);
  return a.status ? MLA_OK : MLA_ERR_CUDA;
}

}  // namespace
}  // namespace vmla

using namespace vmla;

extern "C" {

int mla_paged_check(const mla_paged_cache* cache) { return check_sizes(cache); }

unsigned long long mla_pages_plan_bytes(const mla_paged_cache* cache) {
  return check_sizes(cache) == MLA_OK ? pages_plan_ints(*cache) * sizeof(int) : 0;
}

int mla_pages_resize(mla_paged_cache* cache, const int* new_lens, void* stream) {
  if (!new_lens || !aligned_to(new_lens, 4)) return MLA_ERR_ARG;
  int rc = check_cache(cache, true);
  if (rc == MLA_OK) rc = check_resident({new_lens});
  if (rc != MLA_OK) return rc;
  int* status = device_status_ptr();
  if (!status) return MLA_ERR_CUDA;
  return launch_pages_resize(*cache, new_lens, status, static_cast<cudaStream_t>(stream));
}

int mla_pages_fork(mla_paged_cache* cache, const int* src, const int* dst, int n, void* stream) {
  if (n < 0 || (n > 0 && (!src || !dst)) || !aligned_to(src, 4) || !aligned_to(dst, 4))
    return MLA_ERR_ARG;
  int rc = check_cache(cache, false);
  if (rc == MLA_OK) rc = n > cache->seqs ? MLA_ERR_ARG : check_resident({src, dst});
  if (rc != MLA_OK || n == 0) return rc;
  int* status = device_status_ptr();
  if (!status) return MLA_ERR_CUDA;
  return launch_pages_fork(*cache, src, dst, n, status, static_cast<cudaStream_t>(stream));
}

int mla_pages_copy(mla_paged_cache* cache, const int* src, const int* dst, int n, void* stream) {
  if (n < 0 || (n > 0 && (!src || !dst)) || !aligned_to(src, 4) || !aligned_to(dst, 4))
    return MLA_ERR_ARG;
  int rc = check_cache(cache, false);
  if (rc == MLA_OK) rc = n > cache->pages ? MLA_ERR_ARG : check_resident({src, dst});
  if (rc != MLA_OK || n == 0) return rc;
  int* status = device_status_ptr();
  if (!status) return MLA_ERR_CUDA;
  return launch_pages_copy(*cache, src, dst, n, status, static_cast<cudaStream_t>(stream));
}

int mla_pages_compact(mla_paged_cache* cache, int* new_table, int* new_refs, void* stream) {
  if (!new_table || !new_refs || !aligned_to(new_table, 4) || !aligned_to(new_refs, 4))
    return MLA_ERR_ARG;
  int rc = check_cache(cache, true);
  if (rc == MLA_OK) rc = check_resident({new_table, new_refs});
  if (rc != MLA_OK) return rc;
  int* status = device_status_ptr();
  if (!status) return MLA_ERR_CUDA;
  return launch_pages_compact(*cache, new_table, new_refs, status,
                              static_cast<cudaStream_t>(stream));
}

int mla_paged_append(mla_paged_cache* cache, int layer, const void* c_new, const void* kr_new,
                     int total, const int* q_start, const int* pos, const mla_rope* rope,
                     void* stream) {
  int rc = check_rope(rope);
  if (rc == MLA_OK) rc = check_sizes(cache);
  if (rc != MLA_OK) return rc;
  const int pairs = rope->pairs_t + rope->pairs_h + rope->pairs_w;
  if (layer < 0 || layer >= cache->layers || total < 0 || rope->offset != 0 ||
      2 * pairs != cache->d_r)
    return MLA_ERR_ARG;
  if (total == 0) return check_cache(cache, false);
  if (!c_new || !kr_new || !q_start || !pos || !aligned_to(c_new, 16) ||
      !aligned_to(kr_new, 16) || !aligned_to(q_start, 4) || !aligned_to(pos, 4))
    return MLA_ERR_ARG;
  rc = check_cache(cache, false);
  if (rc == MLA_OK) rc = check_resident({c_new, kr_new, q_start, pos, rope->table});
  if (rc != MLA_OK) return rc;
  const size_t rows = static_cast<size_t>(cache->pages) * cache->page_tokens * layer;
  PagedAppendArgs a;
  a.c_new = c_new;
  a.kr_new = kr_new;
  a.q_start = q_start;
  a.pos = pos;
  a.c = static_cast<char*>(cache->c) + rows * cache->d_c * 2;
  a.kr = static_cast<char*>(cache->kr) + rows * cache->d_r * 2;
  a.table = cache->table;
  a.lens = cache->lens;
  a.rope = static_cast<const float2*>(rope->table);
  a.total = total;
  a.seqs = cache->seqs;
  a.pages = cache->pages;
  a.page_tokens = cache->page_tokens;
  a.max_pages = cache->max_pages;
  a.d_c = cache->d_c;
  a.d_r = cache->d_r;
  a.rope_len = rope->table_len;
  a.pairs_t = rope->pairs_t;
  a.pairs_h = rope->pairs_h;
  a.axes = rope->axes;
  a.layout = rope->layout;
  a.status = device_status_ptr();
  a.stream = static_cast<cudaStream_t>(stream);
  if (!a.status) return MLA_ERR_CUDA;
  return launch_paged_append(a);
}

unsigned long long mla_paged_workspace_bytes(const mla_paged_cache* cache) {
  return check_sizes(cache) == MLA_OK ? paged_attention_workspace(cache->d_c, cache->d_r) : 0;
}

int mla_paged_attention(const mla_paged_cache* cache, int layer, const void* q_c, const void* q_r,
                        int total, int heads, const int* q_start, int head_dim, int causal_block,
                        void* workspace, unsigned long long workspace_bytes, void* o,
                        void* stream) {
  PagedAttnArgs a;
  const int rc = attention_args(cache, layer, q_c, q_r, total, heads, q_start, head_dim,
                                causal_block, workspace, workspace_bytes, o, stream, a);
  if (rc != MLA_OK || total == 0) return rc;
  return launch_paged_attention(a);
}

int mla_paged_window_attention(const mla_paged_cache* cache, const mla_paged_window* window,
                               int layer, const void* q_c, const void* q_r,
                               const void* q_r_sink, int total, int heads, const int* q_start,
                               int head_dim, int causal_block, void* workspace,
                               unsigned long long workspace_bytes, void* o, void* stream) {
  int rc = check_window(window, false);
  if (rc == MLA_OK && !aligned_to(q_r_sink, 16)) rc = MLA_ERR_ARG;
  if (rc != MLA_OK) return rc;
  PagedAttnArgs a;
  rc = attention_args(cache, layer, q_c, q_r, total, heads, q_start, head_dim, causal_block,
                      workspace, workspace_bytes, o, stream, a);
  if (rc == MLA_OK) rc = check_resident({q_r_sink, window->dropped});
  if (rc != MLA_OK || total == 0) return rc;
  a.q_sink = q_r_sink;
  a.dropped = window->dropped;
  a.window = window->window;
  a.sinks = window->sinks;
  return launch_paged_window_attention(a);
}

int mla_selftest_window_form(int form, int* taken) { return window_form(form, taken); }

int mla_paged_window_plan(const mla_paged_cache* cache, const mla_paged_window* window,
                          const int* n_new, int* q_start, int* new_lens, void* stream) {
  if (!n_new || !q_start || !new_lens || !aligned_to(n_new, 4) || !aligned_to(q_start, 4) ||
      !aligned_to(new_lens, 4))
    return MLA_ERR_ARG;
  int rc = check_window(window, false);
  // the metadata calls look up the addresses that they use only: a lookup is a noticeable
  // part of so short a call
  if (rc == MLA_OK) rc = check_buffers(cache, false);
  if (rc == MLA_OK && overlap({{n_new, cache->seqs},
                               {q_start, cache->seqs + 1ll},
                               {new_lens, cache->seqs},
                               {cache->lens, cache->seqs},
                               {window->dropped, cache->seqs}}))
    rc = MLA_ERR_ARG;
  if (rc == MLA_OK)
    rc = check_resident({cache->lens, n_new, q_start, new_lens, window->dropped});
  if (rc != MLA_OK) return rc;
  int* status = device_status_ptr();
  if (!status) return MLA_ERR_CUDA;
  return launch_paged_window_plan(*cache, window->dropped, n_new, q_start, new_lens, status,
                                  static_cast<cudaStream_t>(stream));
}

int mla_paged_window_positions(const mla_paged_cache* cache, const mla_paged_window* window,
                               const int* q_start, int total, int causal_block,
                               int tokens_per_frame, int frame_width, int axes, int* pos,
                               int* pos_sink, int* rows, void* stream) {
  int rc = check_window(window, false);
  if (rc == MLA_OK) rc = check_sizes(cache);
  if (rc != MLA_OK) return rc;
  if (total < 0 || causal_block < 0 || tokens_per_frame < 1 || frame_width < 1 ||
      frame_width > tokens_per_frame || (axes != 1 && axes != 3))
    return MLA_ERR_ARG;
  if (total == 0) return check_cache(cache, false);
  if (!q_start || !pos || !aligned_to(q_start, 4) || !aligned_to(pos, 4) ||
      !aligned_to(pos_sink, 4) || !aligned_to(rows, 4))
    return MLA_ERR_ARG;
  rc = check_buffers(cache, false);
  const long long n = static_cast<long long>(total) * axes;
  if (rc == MLA_OK && overlap({{q_start, cache->seqs + 1ll},
                               {pos, n},
                               {pos_sink, n},
                               {rows, total},
                               {cache->table, table_ints(cache)},
                               {cache->lens, cache->seqs},
                               {window->dropped, cache->seqs}}))
    rc = MLA_ERR_ARG;
  if (rc == MLA_OK)
    rc = check_resident(
        {cache->table, cache->lens, q_start, pos, pos_sink, rows, window->dropped});
  if (rc != MLA_OK) return rc;
  PagedPositionsArgs a;
  a.q_start = q_start;
  a.table = cache->table;
  a.lens = cache->lens;
  a.dropped = window->dropped;
  a.pos = pos;
  a.pos_sink = pos_sink;
  a.rows = rows;
  a.total = total;
  a.seqs = cache->seqs;
  a.pages = cache->pages;
  a.page_tokens = cache->page_tokens;
  a.max_pages = cache->max_pages;
  a.window = window->window;
  a.sinks = window->sinks;
  a.causal_block = causal_block;
  a.tokens_per_frame = tokens_per_frame;
  a.frame_width = frame_width;
  a.axes = axes;
  a.status = device_status_ptr();
  a.stream = static_cast<cudaStream_t>(stream);
  if (!a.status) return MLA_ERR_CUDA;
  return launch_paged_positions(a);
}

int mla_pages_slide(mla_paged_cache* cache, const mla_paged_window* window, const int* keep,
                    void* stream) {
  if (!keep || !aligned_to(keep, 4)) return MLA_ERR_ARG;
  int rc = check_window(window, true);
  if (rc == MLA_OK) rc = check_buffers(cache, false);
  if (rc == MLA_OK && overlap({{cache->table, table_ints(cache)},
                               {cache->lens, cache->seqs},
                               {cache->refs, cache->pages},
                               {keep, cache->seqs},
                               {window->dropped, cache->seqs}}))
    rc = MLA_ERR_ARG;
  if (rc == MLA_OK)
    rc = check_resident({cache->table, cache->lens, cache->refs, keep, window->dropped});
  if (rc != MLA_OK) return rc;
  int* status = device_status_ptr();
  if (!status) return MLA_ERR_CUDA;
  return launch_pages_slide(*cache, *window, keep, status, static_cast<cudaStream_t>(stream));
}

int mla_pages_window_fork(mla_paged_cache* cache, const mla_paged_window* window,
                          const int* src, const int* dst, int n, void* stream) {
  if (n < 0 || (n > 0 && (!src || !dst)) || !aligned_to(src, 4) || !aligned_to(dst, 4))
    return MLA_ERR_ARG;
  int rc = check_window(window, true);
  if (rc == MLA_OK) rc = check_sizes(cache);
  if (rc == MLA_OK && n > cache->seqs) rc = MLA_ERR_ARG;
  if (rc == MLA_OK) rc = check_buffers(cache, false);
  if (rc == MLA_OK)  // src and dst are only read: they may be anywhere else
    for (const int* pairs : {src, dst})
      if (overlap({{cache->table, table_ints(cache)},
                   {cache->lens, cache->seqs},
                   {cache->refs, cache->pages},
                   {pairs, n},
                   {window->dropped, cache->seqs}}))
        rc = MLA_ERR_ARG;
  if (rc == MLA_OK)
    rc = check_resident({cache->table, cache->lens, cache->refs, src, dst, window->dropped});
  if (rc != MLA_OK || n == 0) return rc;
  int* status = device_status_ptr();
  if (!status) return MLA_ERR_CUDA;
  return launch_pages_window_fork(*cache, window->dropped, src, dst, n, status,
                                  static_cast<cudaStream_t>(stream));
}

}  // extern "C"
