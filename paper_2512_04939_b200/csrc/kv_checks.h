// Checks of arguments that the paged K/V cache's entry points share.
#pragma once

#include "kv_cache.h"

namespace lv {

inline bool cache_ok(const litevggt_kv_cache* c) { return c != nullptr && c->magic == kKvCacheMagic; }
inline bool batch_ok(const litevggt_kv_batch* b) { return b != nullptr && b->magic == kKvBatchMagic; }

// A batch of this cache whose arrays are on the device.
inline litevggt_status usable(const litevggt_kv_cache* c, const litevggt_kv_batch* b) {
  if (!cache_ok(c) || b == nullptr) return LITEVGGT_ERR_NULL;
  if (!batch_ok(b) || b->owner_id != c->id || b->base == nullptr) return LITEVGGT_ERR_STALE_PLAN;
  return LITEVGGT_OK;
}

// Rows of heads that may be read 16 bytes at a time.
inline litevggt_status stride_ok(int64_t row, int64_t head) {
  if (row < 0 || head < 0 || row > UINT32_MAX || head > UINT32_MAX) return LITEVGGT_ERR_SHAPE;
  return row % 8 != 0 || head % 8 != 0 ? LITEVGGT_ERR_ALIGN : LITEVGGT_OK;
}

// Whether `n` bytes at `out` reach into one of the rows of queries, each taken from its first head to the end of its last.
inline bool meets_queries(const void* out, long long n, const void* q, long long rows, long long row_bytes, long long row_stride_bytes) {
  const long long begin = (long long)(reinterpret_cast<intptr_t>(out) - reinterpret_cast<intptr_t>(q)), end = begin + n;
  // the first row that ends behind the output's beginning
  long long i = 0;
  if (begin >= row_bytes) {
    if (row_stride_bytes == 0) return false;
    i = (begin - row_bytes) / row_stride_bytes + 1;
  }
  return i < rows && i * row_stride_bytes < end;
}

}  // namespace lv
