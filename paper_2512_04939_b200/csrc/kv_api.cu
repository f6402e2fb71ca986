// The paged K/V cache's entry points: what a batch needs of device memory and how it lies there, the checks of arguments.  Host code only.
#include <string.h>

#include <new>

#include "kv_cache.h"
#include "kv_checks.h"

namespace lv {

namespace {

// Lays out a batch's device memory: first what the host writes (`image`), then what only kernels use.
void lay_out(litevggt_kv_batch* b, const int32_t* pages, size_t n_pages, int head_dim) {
  size_t at = 0;
  auto take = [&](size_t bytes) {
    const size_t here = at;
    at += (size_t)round_up((long long)(bytes > 0 ? bytes : 1), 256);
    return here;
  };
  auto take_lists = [&](const KvWork& w, litevggt_kv_batch::Places* p) {
    p->pieces = take(w.pieces.size() * sizeof(KvPiece));
    p->joins = take((size_t)w.joins * sizeof(int));
    p->again = take(w.pieces.size() * sizeof(int));
  };
  b->o_seqs = take(b->seqs.size() * sizeof(KvSeq));
  b->o_pages = take(n_pages * sizeof(int));
  take_lists(b->few, &b->at_few);
  take_lists(b->tiles, &b->at_tiles);
  b->o_few_at = take(b->weigh.few_at.size() * sizeof(long long));
  b->o_tiles_at = take(b->weigh.tiles_at.size() * sizeof(long long));
  b->o_weigh_joins = take(b->weigh.parts > 1 ? (size_t)b->weigh.items * sizeof(int) : 0);
  b->image.assign(at, 0);  // counters and marks start at zero
  // the two launches follow one another, and so use the same memory
  const size_t parts[2] = {(size_t)b->few.slots * kKvFewRows, (size_t)b->tiles.slots * kKvTileRows};
  const size_t most = std::max(parts[0], parts[1]);
  b->at_few.rows = b->at_tiles.rows = take(most * head_dim * sizeof(float));
  b->at_few.sums = b->at_tiles.sums = take(most * 2 * sizeof(float));
  b->o_weigh_sums = take(b->weigh.parts > 1 ? (size_t)b->weigh.items * b->weigh.parts * b->weigh.key_block * sizeof(float) : 0);
  b->bytes = at;
  auto put = [&](size_t to, const void* from, size_t bytes) {
    if (bytes > 0) memcpy(b->image.data() + to, from, bytes);
  };
  put(b->o_seqs, b->seqs.data(), b->seqs.size() * sizeof(KvSeq));
  put(b->o_pages, pages, n_pages * sizeof(int));
  auto put_lists = [&](const KvWork& w, const litevggt_kv_batch::Places& p) {
    const std::vector<KvPiece> chain = kv_chain(w);
    put(p.pieces, chain.data(), chain.size() * sizeof(KvPiece));
  };
  put(b->o_few_at, b->weigh.few_at.data(), b->weigh.few_at.size() * sizeof(long long));
  put(b->o_tiles_at, b->weigh.tiles_at.data(), b->weigh.tiles_at.size() * sizeof(long long));
  put_lists(b->few, b->at_few);
  put_lists(b->tiles, b->at_tiles);
}

litevggt_status plan_batch(const litevggt_kv_cache* c, int32_t n_seq, const int32_t* rows, const int32_t* lengths, const int32_t* pages,
                           int32_t q_heads, int32_t causal_block, litevggt_kv_batch* b) {
  long long row0 = 0, page0 = 0;
  const bool queries = q_heads != LITEVGGT_KV_NO_QUERIES;
  const long long heads = queries ? q_heads : c->cfg.kv_heads;
  b->rows_held = true;
  for (int i = 0; i < n_seq; ++i) {
    if (rows[i] < 0 || lengths[i] < 0 || lengths[i] > kKvLongest) return LITEVGGT_ERR_SHAPE;
    if (rows[i] > lengths[i]) b->rows_held = false;
    b->seqs.push_back(KvSeq{(int)row0, rows[i], lengths[i], (int)page0});
    row0 += rows[i];
    page0 += ((long long)lengths[i] + c->cfg.page_size - 1) / c->cfg.page_size;
    if (row0 * heads > INT32_MAX || page0 > INT32_MAX) return LITEVGGT_ERR_SHAPE;
  }
  if (page0 > 0 && pages == nullptr) return LITEVGGT_ERR_NULL;
  for (long long i = 0; i < page0; ++i)
    if (pages[i] < 0 || pages[i] >= c->cfg.pages) return LITEVGGT_ERR_SHAPE;
  b->magic = kKvBatchMagic;
  b->owner_id = c->id;
  b->device = c->device;
  b->q_heads = queries ? q_heads : 0;
  b->group = b->q_heads / c->cfg.kv_heads;
  b->causal_block = causal_block;
  b->rows = row0;
  if (!queries) {  // nothing is cut, and no memory kept for parts of rows: 131,072 tokens of 16 heads of 64 would take 1.1 GB of it
    lay_out(b, pages, (size_t)page0, c->cfg.head_dim);
    return LITEVGGT_OK;
  }
  std::vector<int> few, many;
  int most = 0;
  for (int i = 0; i < n_seq; ++i) {
    const long long r = (long long)rows[i] * b->group;
    if (r > kKvFewRows) many.push_back(i);
    else if (r > 0) few.push_back(i), most = std::max(most, (int)r);
  }
  b->few_rows = most;
  const int per_sm = kv_few_ctas(c->cfg.head_dim, c->cfg.dtype != LITEVGGT_KV_BF16);
  b->few = kv_cut(b->seqs, few, b->group, c->cfg.kv_heads, causal_block,
                  KvCut{kKvFewRows, kKvFewUnit, std::min(c->num_sms * per_sm, kKvFewWorkers), kKvFewLeast, INT32_MAX, kKvFewPiece});
  long long keys = 0;
  for (const KvPiece& p : b->few.pieces) keys += p.key1 - p.key0;
  b->few_keys = b->few.pieces.empty() ? 0 : (int)(keys / (long long)b->few.pieces.size());
  // In units of 128 keys against 256 rows.  CTAs of one row tile take more time for the same work, but there are twice as many:
  // where the pieces are few it can be better to have them than to cut keys, since parts have to be joined.
  const double piece = c->cfg.head_dim == 64 ? kKvTilePiece64 : kKvTilePiece128;
  auto cut_tiles = [&](int rows, double unit) {
    KvWork w = kv_cut(b->seqs, many, b->group, c->cfg.kv_heads, causal_block,
                      KvCut{rows, kKvTileUnit, c->num_sms, kKvTileLeast, kKvTileMost, piece / unit});
    w.cost = w.cost * unit + (w.joins > 0 ? kKvJoinCost : 0.0);
    return w;
  };
  b->tiles = cut_tiles(kKvTileRows, 1.0);
  if (b->tiles.cost < kKvShortCost) {  // (elsewhere it cannot win, and need not be counted)
    KvWork narrow = cut_tiles(kKvTileRows / 2, kKvHalfTiles);
    if (narrow.cost < b->tiles.cost) b->tiles = narrow;
  }
  b->weigh = kv_weigh_plan(b->seqs, b->group, c->cfg.kv_heads, kKvFewRows, c->num_sms, c->pool.weights != nullptr);
  lay_out(b, pages, (size_t)page0, c->cfg.head_dim);
  return LITEVGGT_OK;
}

}  // namespace
}  // namespace lv

using namespace lv;

extern "C" {

litevggt_status litevggt_kv_create(const litevggt_kv_config* cfg, int device, void* k, void* v, uint8_t* k_exp, uint8_t* v_exp,
                                   uint32_t* status, litevggt_kv_cache** out) {
  if (cfg == nullptr || out == nullptr) return LITEVGGT_ERR_NULL;
  *out = nullptr;
  if (cfg->head_dim != 64 && cfg->head_dim != 128) return LITEVGGT_ERR_BAD_CONFIG;
  if (cfg->page_size != 16 && cfg->page_size != 32 && cfg->page_size != 64 && cfg->page_size != 128) return LITEVGGT_ERR_BAD_CONFIG;
  if (cfg->dtype != LITEVGGT_KV_BF16 && cfg->dtype != LITEVGGT_KV_E4M3 && cfg->dtype != LITEVGGT_KV_E2M1) return LITEVGGT_ERR_BAD_CONFIG;
  if (cfg->kv_heads < 1 || cfg->pages < 1) return LITEVGGT_ERR_BAD_CONFIG;
  // a row of a head is addressed by one 32-bit coordinate
  if ((long long)cfg->pages * cfg->kv_heads > INT32_MAX / cfg->page_size) return LITEVGGT_ERR_BAD_CONFIG;
  if (k == nullptr || v == nullptr || status == nullptr) return LITEVGGT_ERR_NULL;
  const bool narrow = cfg->dtype != LITEVGGT_KV_BF16;
  if (narrow && (k_exp == nullptr || v_exp == nullptr)) return LITEVGGT_ERR_NULL;
  if (!aligned16(k) || !aligned16(v) || (narrow && (!aligned16(k_exp) || !aligned16(v_exp)))) return LITEVGGT_ERR_ALIGN;
  int count = 0, major = 0, sms = 0;
  if (cudaGetDeviceCount(&count) != cudaSuccess || device < 0 || device >= count) {
    (void)cudaGetLastError();
    return LITEVGGT_ERR_CUDA;
  }
  cudaError_t e = cudaDeviceGetAttribute(&major, cudaDevAttrComputeCapabilityMajor, device);
  if (e == cudaSuccess) e = cudaDeviceGetAttribute(&sms, cudaDevAttrMultiProcessorCount, device);
  if (e != cudaSuccess) return cuda_status(e);
  if (major != 10) return LITEVGGT_ERR_ARCH;
  litevggt_kv_cache* c = new (std::nothrow) litevggt_kv_cache();
  if (c == nullptr) return LITEVGGT_ERR_ALLOC;
  c->magic = kKvCacheMagic;
  c->cfg = *cfg;
  static std::atomic<unsigned long long> made{0};
  c->id = ++made;
  c->device = device;
  c->num_sms = sms;
  int shift = 4;
  while ((1 << shift) < cfg->page_size) ++shift;
  c->pool = KvPool{static_cast<uint8_t*>(k), static_cast<uint8_t*>(v), narrow ? k_exp : nullptr, narrow ? v_exp : nullptr,
                   cfg->kv_heads, cfg->page_size, shift, nullptr};
  c->status = status;
  c->launches = 0;
  if (!narrow) {  // rows of heads as one matrix; a box is a page of a head and 64 channels
    static std::atomic<void*> encode{nullptr};
    void* fn = encode.load(std::memory_order_acquire);
    bool ok = fn != nullptr || resolve_encode_tiled(&fn);
    if (ok) encode.store(fn, std::memory_order_release);
    const uint64_t rows = (uint64_t)cfg->pages * cfg->kv_heads * cfg->page_size, hd = (uint64_t)cfg->head_dim;
    auto make = [&](CUtensorMap* map, const void* base, int box) {
      return make_tmap_bf16_2d(fn, map, base, hd, rows, hd, 64, (uint32_t)box, true);
    };
    ok = ok && make(&c->k_map, k, cfg->page_size) && make(&c->v_map, v, cfg->page_size) && make(&c->k_map16, k, 16) && make(&c->v_map16, v, 16);
    if (!ok) {
      delete c;
      return LITEVGGT_ERR_CUDA;
    }
  }
  *out = c;
  return LITEVGGT_OK;
}

litevggt_status litevggt_kv_destroy(litevggt_kv_cache* cache) {
  if (cache == nullptr) return LITEVGGT_OK;
  if (!cache_ok(cache)) return LITEVGGT_ERR_NULL;
  cache->magic = 0;
  delete cache;
  return LITEVGGT_OK;
}

litevggt_status litevggt_kv_batch_create(const litevggt_kv_cache* cache, int32_t n_seq, const int32_t* rows, const int32_t* lengths,
                                         const int32_t* pages, int32_t q_heads, int32_t causal_block, litevggt_kv_batch** out,
                                         size_t* bytes) {
  if (!cache_ok(cache) || rows == nullptr || lengths == nullptr || out == nullptr || bytes == nullptr) return LITEVGGT_ERR_NULL;
  *out = nullptr;
  if (n_seq < 1 || causal_block < 0) return LITEVGGT_ERR_SHAPE;
  if (q_heads != LITEVGGT_KV_NO_QUERIES && (q_heads < 1 || q_heads % cache->cfg.kv_heads != 0)) return LITEVGGT_ERR_SHAPE;
  litevggt_kv_batch* b = new (std::nothrow) litevggt_kv_batch();
  if (b == nullptr) return LITEVGGT_ERR_ALLOC;
  litevggt_status st = LITEVGGT_ERR_ALLOC;
  try {
    st = plan_batch(cache, n_seq, rows, lengths, pages, q_heads, causal_block, b);
  } catch (...) {  // no memory on the host
  }
  if (st != LITEVGGT_OK) {
    delete b;
    return st;
  }
  *bytes = b->bytes;
  *out = b;
  return LITEVGGT_OK;
}

litevggt_status litevggt_kv_batch_place(litevggt_kv_batch* batch, void* memory, size_t bytes, void* stream) {
  if (!batch_ok(batch) || memory == nullptr) return LITEVGGT_ERR_NULL;
  if (bytes < batch->bytes) return LITEVGGT_ERR_SHAPE;
  if ((reinterpret_cast<uintptr_t>(memory) & 255u) != 0) return LITEVGGT_ERR_ALIGN;
  const OnDevice g(batch->device);
  if (!g.ok) return LITEVGGT_ERR_CUDA;
  // From pageable memory: the call has taken the bytes when it returns.  In a capture it would not have: a graph reads its source
  // again whenever it is replayed, and the batch may be gone by then.
  cudaStreamCaptureStatus capture = cudaStreamCaptureStatusNone;
  cudaError_t e = cudaStreamIsCapturing((cudaStream_t)stream, &capture);
  if (e != cudaSuccess) return cuda_status(e);
  if (capture != cudaStreamCaptureStatusNone) return LITEVGGT_ERR_CUDA;
  e = cudaMemcpyAsync(memory, batch->image.data(), batch->image.size(), cudaMemcpyHostToDevice, (cudaStream_t)stream);
  if (e != cudaSuccess) return cuda_status(e);
  batch->base = static_cast<uint8_t*>(memory);
  return LITEVGGT_OK;
}

litevggt_status litevggt_kv_batch_destroy(litevggt_kv_batch* batch) {
  if (batch == nullptr) return LITEVGGT_OK;
  if (!batch_ok(batch)) return LITEVGGT_ERR_STALE_PLAN;
  batch->magic = 0;
  delete batch;
  return LITEVGGT_OK;
}

litevggt_status litevggt_kv_append(litevggt_kv_cache* cache, const litevggt_kv_batch* batch, const void* k, int64_t k_row_stride,
                                   int64_t k_head_stride, const void* v, int64_t v_row_stride, int64_t v_head_stride, void* stream) {
  litevggt_status st = usable(cache, batch);
  if (st != LITEVGGT_OK) return st;
  if (!batch->rows_held) return LITEVGGT_ERR_SHAPE;
  if (batch->rows == 0) return LITEVGGT_OK;
  if (k == nullptr || v == nullptr) return LITEVGGT_ERR_NULL;
  if (!aligned16(k) || !aligned16(v)) return LITEVGGT_ERR_ALIGN;
  if ((st = stride_ok(k_row_stride, k_head_stride)) != LITEVGGT_OK) return st;
  if ((st = stride_ok(v_row_stride, v_head_stride)) != LITEVGGT_OK) return st;
  const OnDevice g(cache->device);
  if (!g.ok) return LITEVGGT_ERR_CUDA;
  int n = 0;
  const cudaError_t e = launch_kv_append(*cache, *batch, static_cast<const __nv_bfloat16*>(k), KvStride{k_row_stride, k_head_stride},
                                         static_cast<const __nv_bfloat16*>(v), KvStride{v_row_stride, v_head_stride},
                                         (cudaStream_t)stream, &n);
  cache->launches += n;
  return cuda_status(e);
}

litevggt_status litevggt_kv_gather(litevggt_kv_cache* cache, const litevggt_kv_batch* batch, void* k, void* v, void* stream) {
  const litevggt_status st = usable(cache, batch);
  if (st != LITEVGGT_OK) return st;
  if (!batch->rows_held) return LITEVGGT_ERR_SHAPE;
  if (batch->rows == 0) return LITEVGGT_OK;
  if (k == nullptr || v == nullptr) return LITEVGGT_ERR_NULL;
  if (!aligned16(k) || !aligned16(v)) return LITEVGGT_ERR_ALIGN;
  const OnDevice g(cache->device);
  if (!g.ok) return LITEVGGT_ERR_CUDA;
  int n = 0;
  const cudaError_t e =
      launch_kv_gather(*cache, *batch, static_cast<__nv_bfloat16*>(k), static_cast<__nv_bfloat16*>(v), (cudaStream_t)stream, &n);
  cache->launches += n;
  return cuda_status(e);
}

litevggt_status litevggt_kv_attend(litevggt_kv_cache* cache, const litevggt_kv_batch* batch, const void* q, int64_t q_row_stride,
                                   int64_t q_head_stride, float scale, void* out, void* stream) {
  return litevggt_kv_attend_lse(cache, batch, q, q_row_stride, q_head_stride, scale, out, nullptr, stream);
}

litevggt_status litevggt_kv_attend_lse(litevggt_kv_cache* cache, const litevggt_kv_batch* batch, const void* q, int64_t q_row_stride,
                                       int64_t q_head_stride, float scale, void* out, float* lse, void* stream) {
  litevggt_status st = usable(cache, batch);
  if (st != LITEVGGT_OK) return st;
  if (batch->q_heads == 0) return LITEVGGT_ERR_SHAPE;
  if (!(scale > 0.0f) || !(scale < 1e30f)) return LITEVGGT_ERR_SHAPE;
  if (batch->rows == 0) return LITEVGGT_OK;
  if (q == nullptr || out == nullptr) return LITEVGGT_ERR_NULL;
  if (!aligned16(q) || !aligned16(out)) return LITEVGGT_ERR_ALIGN;
  if ((st = stride_ok(q_row_stride, q_head_stride)) != LITEVGGT_OK) return st;
  const long long hd = cache->cfg.head_dim, row_bytes = 2 * ((batch->q_heads - 1) * q_head_stride + hd);
  const long long out_bytes = 2 * batch->rows * batch->q_heads * hd, lse_bytes = 4 * batch->rows * batch->q_heads;
  if (meets_queries(out, out_bytes, q, batch->rows, row_bytes, 2 * q_row_stride)) return LITEVGGT_ERR_SHAPE;
  if (lse != nullptr) {
    if ((reinterpret_cast<uintptr_t>(lse) & 3u) != 0) return LITEVGGT_ERR_ALIGN;
    if (meets_queries(lse, lse_bytes, q, batch->rows, row_bytes, 2 * q_row_stride) || meets_queries(lse, lse_bytes, out, 1, out_bytes, 0))
      return LITEVGGT_ERR_SHAPE;
  }
  const OnDevice g(cache->device);
  if (!g.ok) return LITEVGGT_ERR_CUDA;
  const KvAttend a{static_cast<const __nv_bfloat16*>(q), KvStride{q_row_stride, q_head_stride}, static_cast<__nv_bfloat16*>(out),
                   batch->q_heads, batch->group, batch->causal_block, scale * 1.4426950408889634f, lse};
  int n = 0;
  cudaError_t e = cudaSuccess;
  if (!batch->few.pieces.empty()) e = launch_kv_attn_few(*cache, *batch, a, (cudaStream_t)stream, &n);
  if (e == cudaSuccess && !batch->tiles.pieces.empty()) e = launch_kv_attn_tiles(*cache, *batch, a, (cudaStream_t)stream, &n);
  cache->launches += n;
  return cuda_status(e);
}

litevggt_status litevggt_kv_poll(litevggt_kv_cache* cache, void* stream) {
  if (!cache_ok(cache)) return LITEVGGT_ERR_NULL;
  const OnDevice g(cache->device);
  if (!g.ok) return LITEVGGT_ERR_CUDA;
  cudaStream_t s = (cudaStream_t)stream;
  uint32_t word = 0;
  cudaError_t e = cudaMemcpyAsync(&word, cache->status, sizeof(word), cudaMemcpyDeviceToHost, s);
  if (e == cudaSuccess) e = cudaMemsetAsync(cache->status, 0, sizeof(word), s);
  if (e == cudaSuccess) e = cudaStreamSynchronize(s);
  if (e != cudaSuccess) return cuda_status(e);
  return word & kStatusTimeout ? LITEVGGT_ERR_DEVICE_TIMEOUT : LITEVGGT_OK;
}

litevggt_status litevggt_kv_launch_count(const litevggt_kv_cache* cache, int64_t* launches) {
  if (!cache_ok(cache) || launches == nullptr) return LITEVGGT_ERR_NULL;
  *launches = cache->launches;
  return LITEVGGT_OK;
}

}  // extern "C"
