// The entry points of tallies and eviction: the checks of arguments.  Host code only.
#include <string.h>

#include "kv_checks.h"

namespace lv {
namespace {

// Whether no page of the batch's list is named twice.  Looked up once: a batch's pages do not change.
bool pages_apart(const litevggt_kv_cache& c, const litevggt_kv_batch& b) {
  int apart = b.pages_apart;
  if (apart < 0) {
    std::vector<bool> seen((size_t)c.cfg.pages, false);
    const int* pages = kv_host_pages(b);
    apart = 1;
    for (long long i = 0, n = kv_page_count(b, c.cfg.page_size); i < n && apart; ++i) {
      if (seen[(size_t)pages[i]]) apart = 0;
      seen[(size_t)pages[i]] = true;
    }
    b.pages_apart = apart;
  }
  return apart != 0;
}

bool pages_meet(const litevggt_kv_cache& c, const litevggt_kv_batch& a, const litevggt_kv_batch& b) {
  std::vector<bool> seen((size_t)c.cfg.pages, false);
  const int *of_a = kv_host_pages(a), *of_b = kv_host_pages(b);
  for (long long i = 0, n = kv_page_count(a, c.cfg.page_size); i < n; ++i) seen[(size_t)of_a[i]] = true;
  for (long long i = 0, n = kv_page_count(b, c.cfg.page_size); i < n; ++i)
    if (seen[(size_t)of_b[i]]) return true;
  return false;
}

}  // namespace
}  // namespace lv

using namespace lv;

extern "C" {

litevggt_status litevggt_kv_track(litevggt_kv_cache* cache, float* weights) {
  if (!cache_ok(cache)) return LITEVGGT_ERR_NULL;
  if (!aligned16(weights)) return LITEVGGT_ERR_ALIGN;
  cache->pool.weights = weights;
  return LITEVGGT_OK;
}

litevggt_status litevggt_kv_weigh(litevggt_kv_cache* cache, const litevggt_kv_batch* batch, const void* q, int64_t q_row_stride,
                                  int64_t q_head_stride, float scale, const float* lse, float decay, void* stream) {
  litevggt_status st = usable(cache, batch);
  if (st != LITEVGGT_OK) return st;
  if (cache->pool.weights == nullptr) return LITEVGGT_ERR_NULL;
  if (batch->q_heads == 0) return LITEVGGT_ERR_SHAPE;
  if (!(scale > 0.0f) || !(scale < 1e30f) || !(decay >= 0.0f) || !(decay <= 1.0f)) return LITEVGGT_ERR_SHAPE;
  if (batch->rows == 0) return LITEVGGT_OK;
  if (q == nullptr || lse == nullptr) return LITEVGGT_ERR_NULL;
  if (!aligned16(q) || (reinterpret_cast<uintptr_t>(lse) & 3u) != 0) return LITEVGGT_ERR_ALIGN;
  if ((st = stride_ok(q_row_stride, q_head_stride)) != LITEVGGT_OK) return st;
  try {
    if (!pages_apart(*cache, *batch)) return LITEVGGT_ERR_SHAPE;
  } catch (...) {  // no memory on the host
    return LITEVGGT_ERR_ALLOC;
  }
  const OnDevice g(cache->device);
  if (!g.ok) return LITEVGGT_ERR_CUDA;
  const KvWeighing w{static_cast<const __nv_bfloat16*>(q), KvStride{q_row_stride, q_head_stride}, lse, batch->q_heads, batch->group,
                     batch->causal_block, scale * 1.4426950408889634f, decay};
  int n = 0;
  cudaError_t e = launch_kv_weigh_few(*cache, *batch, w, (cudaStream_t)stream, &n);
  if (e == cudaSuccess) e = launch_kv_weigh_tiles(*cache, *batch, w, (cudaStream_t)stream, &n);
  cache->launches += n;
  return cuda_status(e);
}

litevggt_status litevggt_kv_evict(litevggt_kv_cache* cache, const litevggt_kv_batch* from, const litevggt_kv_batch* into, int32_t first,
                                  int32_t last, int32_t* kept, void* stream) {
  litevggt_status st = usable(cache, from);
  if (st != LITEVGGT_OK) return st;
  if ((st = usable(cache, into)) != LITEVGGT_OK) return st;
  if (cache->pool.weights == nullptr) return LITEVGGT_ERR_NULL;
  if (first < 0 || last < 0 || from->seqs.size() != into->seqs.size()) return LITEVGGT_ERR_SHAPE;
  long long most = 0;
  for (size_t i = 0; i < from->seqs.size(); ++i) {
    const KvSeq &a = from->seqs[i], &b = into->seqs[i];
    if (b.rows != b.len || b.len > a.len || (b.len < a.len && (long long)first + last > b.len)) return LITEVGGT_ERR_SHAPE;
    most += b.len;
  }
  if (most == 0) return LITEVGGT_OK;
  if ((long long)from->seqs.size() * cache->cfg.kv_heads > INT32_MAX / 16) return LITEVGGT_ERR_SHAPE;
  if (kept == nullptr) return LITEVGGT_ERR_NULL;
  if ((reinterpret_cast<uintptr_t>(kept) & 3u) != 0) return LITEVGGT_ERR_ALIGN;
  try {
    if (!pages_apart(*cache, *into) || pages_meet(*cache, *from, *into)) return LITEVGGT_ERR_SHAPE;
  } catch (...) {  // no memory on the host
    return LITEVGGT_ERR_ALLOC;
  }
  const OnDevice g(cache->device);
  if (!g.ok) return LITEVGGT_ERR_CUDA;
  int n = 0;
  const cudaError_t e = launch_kv_evict(*cache, *from, *into, first, last, kept, (cudaStream_t)stream, &n);
  cache->launches += n;
  return cuda_status(e);
}

}  // extern "C"
