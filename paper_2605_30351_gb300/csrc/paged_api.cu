// C ABI of the paged latent cache: argument checks and dispatch. See
// include/videomla.h.
#include <cmath>

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

// The cache's own buffers, for an operation that needs the plan or not.
int check_cache(const mla_paged_cache* c, bool plan) {
  const int rc = check_sizes(c);
  if (rc != MLA_OK) return rc;
  if (!c->c || !c->kr || !c->table || !c->lens || !c->refs || (plan && !c->plan))
    return MLA_ERR_ARG;
  if (!aligned_to(c->c, 16) || !aligned_to(c->kr, 16) || !aligned_to(c->table, 16) ||
      !aligned_to(c->lens, 16) || !aligned_to(c->refs, 16) || !aligned_to(c->plan, 16))
    return MLA_ERR_ARG;
  return check_resident({c->c, c->kr, c->table, c->lens, c->refs, plan ? c->plan : nullptr});
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
  int rc = check_sizes(cache);
  if (rc != MLA_OK) return rc;
  if (layer < 0 || layer >= cache->layers || total < 0 || heads < 1 || head_dim < 1 ||
      causal_block < 0 || static_cast<long long>(total) * heads > (1ll << 30))
    return MLA_ERR_ARG;
  const unsigned long long need = paged_attention_workspace(cache->d_c, cache->d_r);
  if (need == 0) return MLA_ERR_UNSUPPORTED;
  if (total == 0) return check_cache(cache, false);
  if (!q_c || !q_r || !q_start || !workspace || !o || !aligned_to(q_c, 16) ||
      !aligned_to(q_r, 16) || !aligned_to(q_start, 4) || !aligned_to(workspace, 16) ||
      !aligned_to(o, 16) || workspace_bytes < need)
    return MLA_ERR_ARG;
  rc = check_cache(cache, false);
  if (rc == MLA_OK) rc = check_resident({q_c, q_r, q_start, workspace, o});
  if (rc != MLA_OK) return rc;
  const size_t rows = static_cast<size_t>(cache->pages) * cache->page_tokens * layer;
  PagedAttnArgs a;
  a.q_c = q_c;
  a.q_r = q_r;
  a.q_start = q_start;
  a.c = static_cast<char*>(cache->c) + rows * cache->d_c * 2;
  a.kr = static_cast<char*>(cache->kr) + rows * cache->d_r * 2;
  a.table = cache->table;
  a.lens = cache->lens;
  a.workspace = workspace;
  a.o = o;
  a.total = total;
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
  if (!a.status) return MLA_ERR_CUDA;
  return launch_paged_attention(a);
}

}  // extern "C"
