// The objects behind the paged K/V cache's entry points, and what its kernels are launched with.
#pragma once

#include <atomic>
#include <vector>

#include "host_common.h"
#include "kv_plan.h"

namespace lv {

constexpr uint32_t kKvCacheMagic = 0x4c564b43u;
constexpr uint32_t kKvBatchMagic = 0x4c564b42u;
constexpr int kKvLongest = 1 << 30;  // tokens of a sequence: sums of positions and steps stay inside 31 bits

// The pools as a kernel sees them: [pages, kv_heads, page_size, head_dim] of bf16 or E4M3 codes, the codes' exponents
// [pages, kv_heads, page_size]; E2M1 codes two to a byte, their exponents [.., head_dim / 32].
struct KvPool {
  uint8_t *k, *v;
  uint8_t *k_exp, *v_exp;  // null for bf16
  int kv_heads, page_size, page_shift;
  float* weights;          // [pages, kv_heads, page_size], what tokens have drawn of the attention; or null
};

// A batch's arrays on the device.
struct KvArrays {
  const KvSeq* seqs;
  const int* pages;
  int n_seq;
};
struct KvLaunch {
  const KvPiece* pieces;
  int workers;
  int* joins;   // counters, zero between launches
  int* again;   // marks of the pieces, likewise
  float* rows;  // partial rows, as the kernel lays them out
  float* sums;  // their {reference, sum}
};

// Rows of a tensor [rows, heads, head_dim]: elements from one row to the next, from one head to the next.
struct KvStride {
  long long row, head;
};

struct KvAttend {
  const __nv_bfloat16* q;
  KvStride q_stride;
  __nv_bfloat16* out;  // [rows, q_heads, head_dim]
  int q_heads, group, causal_block;
  float scale_log2;    // softmax scale in base-2 units
  float* lse;          // [rows, q_heads] natural logarithms of the rows' sums, or null
  // the row's, whose sum of 2^(score - reference) is `sum`
#ifdef __CUDACC__
  __device__ __forceinline__ void put_lse(long long row, bool sees, float reference, float sum) const {
    lse[row] = sees ? (reference + log2f(sum)) * 0.6931471805599453f : -INFINITY;
  }
#endif
};
}  // namespace lv

struct litevggt_kv_cache {
  uint32_t magic;
  unsigned long long id;  // no two caches of a process have the same (their addresses may come round)
  litevggt_kv_config cfg;
  int device, num_sms;
  lv::KvPool pool;
  uint32_t* status;
  CUtensorMap k_map, v_map;      // bf16 pools, boxes of one page of a head and 64 channels
  CUtensorMap k_map16, v_map16;  // the same in boxes of 16 tokens
  long long launches;
};

struct litevggt_kv_batch {
  uint32_t magic;
  unsigned long long owner_id;  // of the cache whose pool its page numbers were checked against
  int device;
  int q_heads, group, causal_block;
  long long rows;
  bool rows_held;  // no sequence has more rows than tokens
  std::vector<lv::KvSeq> seqs;
  lv::KvWork few, tiles;       // sequences of few rows, and the others
  int few_rows;                // the most of the former
  int few_keys;                // of a piece of theirs, on average
  lv::KvWeigh weigh;
  mutable std::atomic<int> pages_apart{-1};  // whether no page is named twice; -1: nobody has looked (calls may do so at once)
  std::vector<uint8_t> image;  // what the device gets
  size_t bytes;                // of device memory
  size_t o_seqs, o_pages;
  struct Places {
    size_t pieces, joins, again, rows, sums;
  } at_few, at_tiles;
  size_t o_few_at, o_tiles_at, o_weigh_joins, o_weigh_sums;
  uint8_t* base = nullptr;     // the caller's device memory
};

namespace lv {

inline KvArrays kv_arrays(const litevggt_kv_batch& b) {
  return KvArrays{reinterpret_cast<const KvSeq*>(b.base + b.o_seqs), reinterpret_cast<const int*>(b.base + b.o_pages), (int)b.seqs.size()};
}

inline KvLaunch kv_launch(const litevggt_kv_batch& b, const KvWork& work, const litevggt_kv_batch::Places& at) {
  return KvLaunch{reinterpret_cast<const KvPiece*>(b.base + at.pieces), work.workers(), reinterpret_cast<int*>(b.base + at.joins), reinterpret_cast<int*>(b.base + at.again),
                  reinterpret_cast<float*>(b.base + at.rows), reinterpret_cast<float*>(b.base + at.sums)};
}

inline long long kv_page_count(const litevggt_kv_batch& b, int page_size) {
  return b.seqs.back().page0 + ((long long)b.seqs.back().len + page_size - 1) / page_size;
}
inline const int* kv_host_pages(const litevggt_kv_batch& b) { return reinterpret_cast<const int*>(b.image.data() + b.o_pages); }

// kv_cache.cu
cudaError_t launch_kv_append(const litevggt_kv_cache& c, const litevggt_kv_batch& b, const __nv_bfloat16* k, KvStride k_stride,
                             const __nv_bfloat16* v, KvStride v_stride, cudaStream_t s, int* launches);
cudaError_t launch_kv_gather(const litevggt_kv_cache& c, const litevggt_kv_batch& b, __nv_bfloat16* k, __nv_bfloat16* v, cudaStream_t s,
                             int* launches);

// kv_attn_few.cu
constexpr int kKvFewRows = 16;    // rows of a piece at most
constexpr int kKvFewWarps = 8;
constexpr int kKvFewUnit = 128;   // keys
// A piece of so many units at least where keys are cut, and what a piece costs beside its keys: a token over 262 keys takes
// 8.2 us in one CTA a head, 4.9 in two, over 1,041 9.0 and 8.5, over 4,164 11.6 and 9.0 (least 4 and 2; eight are worse everywhere).
constexpr int kKvFewLeast = 2;
constexpr double kKvFewPiece = 1.5;
constexpr int kKvFewWorkers = 512;  // CTAs of a launch at most: the weights of a row's parts lie in shared memory
int kv_few_ctas(int head_dim, bool narrow);  // on an SM
cudaError_t launch_kv_attn_few(const litevggt_kv_cache& c, const litevggt_kv_batch& b, const KvAttend& a, cudaStream_t s, int* launches);
// kv_attn_tiles.cu
constexpr int kKvTileRows = 256;
constexpr int kKvTileUnit = 128;
// Units of a piece: at least, where keys are cut; at most, so that no accumulator is carried through more than 512 tiles
// (the tensor core's chain of additions loses bits that sums in 32 bits between pieces keep).
constexpr int kKvTileLeast = 4, kKvTileMost = 512;
// What a piece costs beside its keys, joining its parts, a unit of half the rows, in units (measured on 261 rows over 522 keys up to
// 2,748 over 21,984): 1,041 rows over 5,205 keys 48.1 us with 4 for a piece, 45.5 with 2; chunks of head dim 128 the other
// way about, 278 and 256 us, their rows being twice as long.  261 rows over 522 keys: 15.0 us in tiles of two, 14.0 in single ones.
constexpr double kKvTilePiece64 = 2.0, kKvTilePiece128 = 4.0, kKvJoinCost = 8.0, kKvHalfTiles = 0.8, kKvShortCost = 200.0;
cudaError_t launch_kv_attn_tiles(const litevggt_kv_cache& c, const litevggt_kv_batch& b, const KvAttend& a, cudaStream_t s, int* launches);
// kv_weigh.cu
struct KvWeighing {
  const __nv_bfloat16* q;
  KvStride q_stride;
  const float* lse;  // [rows, q_heads]
  int q_heads, group, causal_block;
  float scale_log2, decay;
};
cudaError_t launch_kv_weigh_few(const litevggt_kv_cache& c, const litevggt_kv_batch& b, const KvWeighing& w, cudaStream_t s, int* launches);
cudaError_t launch_kv_weigh_tiles(const litevggt_kv_cache& c, const litevggt_kv_batch& b, const KvWeighing& w, cudaStream_t s, int* launches);
// kv_evict.cu
cudaError_t launch_kv_evict(const litevggt_kv_cache& c, const litevggt_kv_batch& from, const litevggt_kv_batch& into, int first, int last,
                            int* kept, cudaStream_t s, int* launches);

}  // namespace lv
