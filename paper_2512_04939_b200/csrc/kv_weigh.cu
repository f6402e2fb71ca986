// What cached tokens draw of the attention of a batch's rows, given each row's log-sum-exp:
//   w_j = decay w_j + sum_i p_ij,   p_ij = 2^(c q_i k_j - l_i)  for the rows i that see the key j
// Nothing is multiplied by V, and a key's sum runs over rows, so the scores are taken with keys as the product's rows: a thread owns a
// key, adds along its own row and needs nobody else's numbers.  What a row does not see is left out by a comparison, so nothing that
// lies there has any influence.
//
// Few rows are bound by K's bytes: 16 tokens of 32 heads on 4 over up to 8,328 keys of 128 channels in 8 bits (45 MB) 13 us where the codes
// are still in L2 and 17 where they come from memory, by the latency of a unit's loads (18.6 us before units were fetched two ahead and codes
// became f16 operands); one token over 262 4.5 us; one over 520,500 in bf16 182 us, 6.0 TB/s, and 219 where the tallies that are there are read as
// well (a decay other than zero).  Chunks are bound by exponentials, see there.
#include "exp2.cuh"
#include "kv_cache.h"
#include "kv_mma.cuh"
#include "kv_quant.cuh"

namespace lv {

namespace {

constexpr float kLog2e = 1.4426950408889634f;

// 16 bytes to shared memory, or zeros.
__device__ __forceinline__ void cp_async16(uint8_t* dst, const void* src, bool there) {
  asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(smem_u32(dst)), "l"(src), "r"(there ? 16 : 0) : "memory");
}
__device__ __forceinline__ void cp_async_commit() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int kPending>
__device__ __forceinline__ void cp_async_wait() { asm volatile("cp.async.wait_group %0;" ::"n"(kPending) : "memory"); }

// What a launch over either kind of sequence is given.
struct WeighLists {
  const long long* at;  // units or items of a head before each sequence
  int parts;
  int* joins;
  float* sums;
};

// The sequence that number n of all heads' units belongs to: the last one that begins at or before it (ones without units share their
// successor's start).  The whole warp looks, 32 at a time.
__device__ __forceinline__ int seq_of_unit(const long long* at, int n_seq, int heads, long long n) {
  const int lane = threadIdx.x & 31;
  int found = 0;
  for (int base = 0; base < n_seq; base += 32) {
    const bool begun = base + lane < n_seq && at[base + lane] * heads <= n;
    const uint32_t those = __ballot_sync(0xffffffffu, begun);
    if (those == 0u) break;
    found = base + 31 - __clz(those);
  }
  return found;
}

__device__ __forceinline__ float tallied(float decay, float before, float sum) { return decay == 0.0f ? sum : fmaf(decay, before, sum); }

// ------------------------------------------------------------------ few rows
// A warp's unit is 32 keys of a head, whose K rows it loads straight into the fragments of mma.m16n8k16 with Q as the other operand:
// the four lanes of a key read its row in 16 bytes each (or a quarter row each), and the contraction runs over the channels in that order.
// HBM bounds it: K once, 4 operations a byte at one row; a unit's 4 KB are all under way at once.
constexpr int kWeighWarps = 4;

template <int kHd, int kKind>
struct FewKeys {
  static constexpr int kRowBytes = KvRow<kHd, kKind>::kBytes, kExps = KvRow<kHd, kKind>::kExps;
  static constexpr int kRun = kKind == LITEVGGT_KV_E4M3 ? 16 : 8;  // channels side by side in a lane
  static constexpr int kWords = kRowBytes / 16;  // of a lane: a quarter of the row
  static constexpr int kBlocks = kWords == 16 ? 2 : kHd == 128 ? 3 : 4;  // on an SM: registers
  uint32_t w[4][kWords];                         // of the keys lane / 4 of four tiles of 8
  static constexpr int kExpWords = kExps > 2 ? kExps / 2 : 1;
  uint32_t exps[4][kExpWords];  // of the keys 2 (lane % 4) and the next one of each tile
};

// Where a warp is in its run: a head's unit, and the pages that its first and its second 16 keys lie in.
struct FewPlace {
  KvSeq seq;
  int s, head, key0;
  int page[2];
  __device__ __forceinline__ void look_up(const KvPool& pool, const KvArrays& arrays) {
#pragma unroll
    for (int h = 0; h < 2; ++h)  // (of a second half that is not there the first's)
      page[h] = arrays.pages[seq.page0 + (min(key0 + 16 * h, seq.len - 1) >> pool.page_shift)];
  }
  __device__ __forceinline__ size_t row(const KvPool& pool, int h) const {  // of the pool
    const int key = min(key0 + 16 * h, seq.len - 1) & ~15;
    return (((size_t)page[h] * pool.kv_heads + head) << pool.page_shift) + (key & (pool.page_size - 1));
  }
  // The next keys, the next head, or the next sequence that has units; there is one.
  __device__ __forceinline__ void advance(const KvPool& pool, const KvArrays& arrays, const long long* at) {
    key0 += kKvWeighUnit;
    if (key0 >= seq.len) {
      key0 = 0;
      if (++head == pool.kv_heads) {
        head = 0;
        do ++s;
        while (at[s + 1] == at[s]);
        seq = arrays.seqs[s];
      }
    }
    look_up(pool, arrays);
  }
};

template <int kHd, int kKind, bool kHalf>
__global__ void __launch_bounds__(kWeighWarps * 32, (FewKeys<kHd, kKind>::kBlocks))
kv_weigh_few_kernel(KvPool pool, KvArrays arrays, KvWeighing in, WeighLists lists, long long per_warp, long long units) {
  using Keys = FewKeys<kHd, kKind>;
  constexpr int kHalves = kHalf ? 1 : 2, kRun = Keys::kRun, kSteps = kHd / 16;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, g = lane >> 2, q4 = lane & 3;
  long long unit = ((long long)blockIdx.x * kWeighWarps + warp) * per_warp;
  const long long end = min(unit + per_warp, units);
  // Three units are under way: one is worked on, of the next the keys are, of the one behind it the pages' numbers.
  // (a batch's arrays were there before whatever kernel is still running)
  FewPlace place, ahead;
  if (unit < end) {
    place.s = seq_of_unit(lists.at, arrays.n_seq, pool.kv_heads, unit);
    const long long in_head = lists.at[place.s + 1] - lists.at[place.s], rest = unit - lists.at[place.s] * pool.kv_heads;
    place.head = (int)(rest / in_head);
    place.key0 = (int)(rest % in_head) * kKvWeighUnit;
    place.seq = arrays.seqs[place.s];
    place.look_up(pool, arrays);
    ahead = place;
    if (unit + 1 < end) ahead.advance(pool, arrays, lists.at);
  }
  wait_for_previous_kernel();
  if (unit >= end) return;
  auto load = [&](Keys& k, const FewPlace& p) {
#pragma unroll
    for (int t = 0; t < 4; ++t) {
      const size_t row0 = p.row(pool, t >> 1) + 8 * (t & 1);
      const uint8_t* src = pool.k + (row0 + g) * Keys::kRowBytes;
      if constexpr (kKind == LITEVGGT_KV_E2M1) {
#pragma unroll
        for (int i = 0; i < Keys::kWords; ++i) k.w[t][i] = *reinterpret_cast<const uint32_t*>(src + i * 16 + q4 * 4);
      } else {
#pragma unroll
        for (int i = 0; i < Keys::kWords / 4; ++i) {
          const uint4 x = ldg16(src + (i * 4 + q4) * 16);
          k.w[t][4 * i] = x.x, k.w[t][4 * i + 1] = x.y, k.w[t][4 * i + 2] = x.z, k.w[t][4 * i + 3] = x.w;
        }
      }
      if constexpr (Keys::kExps > 0) {
        const uint8_t* at = pool.k_exp + (row0 + 2 * q4) * Keys::kExps;
        if constexpr (Keys::kExps == 1) {
          k.exps[t][0] = *reinterpret_cast<const uint16_t*>(at);
        } else {
#pragma unroll
          for (int i = 0; i < Keys::kExpWords; ++i) k.exps[t][i] = reinterpret_cast<const uint32_t*>(at)[i];
        }
      }
    }
  };
  Keys k, k_ahead;
  load(k, place);
  bool fresh = true;
  uint32_t qa[kSteps][2 * kHalves];
  float less[kHalves];  // the rows' log-sum-exp in base 2
  float row_scale[kHalves];
  constexpr bool kCodes = kKind != LITEVGGT_KV_BF16;  // their products are of f16, the powers of two stay outside
  constexpr int kBlocks = kKind == LITEVGGT_KV_E2M1 ? kHd / 32 : 1;
  int seen[kHalves];
  for (; unit < end; ++unit) {
    FewPlace behind = ahead;
    if (unit + 1 < end) load(k_ahead, ahead);
    if (unit + 2 < end) behind.advance(pool, arrays, lists.at);
    if (fresh) {  // the rows
      const KvSeq& seq = place.seq;
      const int rows = seq.rows * in.group;
#pragma unroll
      for (int half = 0; half < kHalves; ++half) {
        const int r = g + 8 * half;
        const bool live = r < rows;
        const int token = live ? r / in.group : 0, q_head = place.head * in.group + (live ? r % in.group : 0);
        const __nv_bfloat16* src = in.q + (seq.row0 + token) * in.q_stride.row + q_head * in.q_stride.head;
#pragma unroll
        for (int i = 0; i < kHd / (4 * kRun); ++i)
#pragma unroll
          for (int j = 0; j < kRun / 4; ++j) {
            const uint2 x = live ? *reinterpret_cast<const uint2*>(src + (i * 4 + q4) * kRun + 4 * j) : make_uint2(0u, 0u);
            qa[i * (kRun / 4) + j][half] = x.x;
            qa[i * (kRun / 4) + j][kHalves + half] = x.y;
          }
        row_scale[half] = in.scale_log2;
        if constexpr (kCodes) {
          uint32_t top = 0;
#pragma unroll
          for (int i = 0; i < kSteps; ++i) top = __vmaxu2(top, __vmaxu2(qa[i][half] & 0x7fff7fffu, qa[i][kHalves + half] & 0x7fff7fffu));
          top = max(top & 0xffffu, top >> 16);
          top = max(top, __shfl_xor_sync(0xffffffffu, top, 1));
          top = max(top, __shfl_xor_sync(0xffffffffu, top, 2));
          const float2 factors = f16_factor(top);
          row_scale[half] *= factors.y;
#pragma unroll
          for (int i = 0; i < kSteps; ++i)
#pragma unroll
            for (int j = 0; j < 2; ++j) {
              const uint32_t x = qa[i][j * kHalves + half];
              qa[i][j * kHalves + half] = pack_f16(bf16_lo(x) * factors.x, bf16_hi(x) * factors.x);
            }
        }
        less[half] = live ? -kLog2e * in.lse[(long long)(seq.row0 + token) * in.q_heads + q_head] : 0.0f;
        seen[half] = live ? kv_seen(seq.len, seq.rows, in.causal_block, token) : 0;
      }
    }
    const int key0 = place.key0;
    float drawn[4][2];  // of the keys 2 q4 and 2 q4 + 1 of each tile, over this lane's rows
#pragma unroll
    for (int t = 0; t < 4; ++t) {
      float c[kBlocks][4];
#pragma unroll
      for (int b = 0; b < kBlocks; ++b) c[b][0] = c[b][1] = c[b][2] = c[b][3] = 0.0f;
      auto step = [&](int n, uint32_t b0, uint32_t b1) {
        float (&to)[4] = c[kBlocks > 1 ? n / 2 : 0];
        if constexpr (kHalf) mma_16816<kCodes>(to, qa[n][0], 0u, qa[n][1], 0u, b0, b1);
        else mma_16816<kCodes>(to, qa[n][0], qa[n][kHalves - 1], qa[n][kHalves], qa[n][2 * kHalves - 1], b0, b1);
      };
      float power[kCodes ? 4 * Keys::kExpWords : 1];  // of the two keys, block by block
      if constexpr (kKind == LITEVGGT_KV_BF16) {
#pragma unroll
        for (int n = 0; n < kSteps; ++n) step(n, k.w[t][2 * n], k.w[t][2 * n + 1]);
      } else if constexpr (kKind == LITEVGGT_KV_E4M3) {
#pragma unroll
        for (int n = 0; n < kSteps; ++n) step(n, widen_low(k.w[t][n]), widen_high(k.w[t][n]));
      } else {
#pragma unroll
        for (int i = 0; i < kBlocks; ++i) {
          uint32_t x[4];
          widen_codes4(k.w[t][i], x);
          step(2 * i, x[0], x[1]);
          step(2 * i + 1, x[2], x[3]);
        }
      }
      if constexpr (kCodes) {
#pragma unroll
        for (int i = 0; i < Keys::kExpWords; ++i) power_word(k.exps[t][i], *reinterpret_cast<float (*)[4]>(&power[4 * i]));
      }
#pragma unroll
      for (int e = 0; e < 2; ++e) {
        const int key = key0 + 8 * t + 2 * q4 + e;
        drawn[t][e] = 0.0f;
#pragma unroll
        for (int half = 0; half < kHalves; ++half) {
          float x = less[half];
#pragma unroll
          for (int b = 0; b < kBlocks; ++b) {
            const float y = c[b][2 * half + e];
            x = kCodes ? fmaf(y * row_scale[half], power[kCodes ? e * kBlocks + b : 0], x) : fmaf(y, row_scale[half], x);
          }
          const float p = fast_exp2(x);
          if (key < seen[half]) drawn[t][e] += p;
        }
      }
    }
    // Over the eight lanes that hold other rows of the same keys; each of the 32 ends with one key.
    float two[2][2];
#pragma unroll
    for (int h = 0; h < 2; ++h)
#pragma unroll
      for (int e = 0; e < 2; ++e) {
        const bool upper = (lane & 16) != 0;
        const float own = upper ? drawn[2 * h + 1][e] : drawn[2 * h][e], other = upper ? drawn[2 * h][e] : drawn[2 * h + 1][e];
        two[h][e] = own + __shfl_xor_sync(0xffffffffu, other, 16);
      }
    float one[2];
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      const bool upper = (lane & 8) != 0;
      const float own = upper ? two[h][1] : two[h][0], other = upper ? two[h][0] : two[h][1];
      one[h] = own + __shfl_xor_sync(0xffffffffu, other, 8);
    }
    const bool upper = (lane & 4) != 0;
    const float own = upper ? one[1] : one[0], other = upper ? one[0] : one[1];
    const float sum = own + __shfl_xor_sync(0xffffffffu, other, 4);
    const int in16 = 8 * (lane >> 4) + 2 * q4 + ((lane >> 3) & 1);
    if (key0 + 16 * (upper ? 1 : 0) + in16 < place.seq.len) {
      float* w = pool.weights + place.row(pool, upper ? 1 : 0) + in16;
      *w = tallied(in.decay, in.decay == 0.0f ? 0.0f : *w, sum);
    }
    fresh = ahead.s != place.s || ahead.head != place.head;
    place = ahead;
    ahead = behind;
    k = k_ahead;
  }
}

// ------------------------------------------------------------------ chunks
// Scores on the 5th-generation tensor cores, 128 keys by 128 rows a product, kTiles of them side by side against the same rows.  One
// exponential a score and 64 (128) multiplications for it, so the special-function unit is the bound, at 16 a clock; the products need
// an eighth (a quarter) of its time.  Roles: eight warps take the exponentials, each thread a key against all rows or a share of them; one
// issues the products; one fetches K once an item, by TMA, or two widen its codes; four fetch Q tile by tile into swizzled shared memory,
// with what the exponentials need of a row, its log-sum-exp and how many keys it sees; and one
// finds out what the CTA's items are, 32 at a time and ahead of all others: the divisions and searches of that, thousands of clocks in a
// row, were half of the time of short items.
// 4164 rows over 41,640 keys, 16 heads of 64: 798 us, 3.3 10^12 exponentials a second, four fifths of what the unit gives at the clock held
// (1.76 GHz).  Tried and left: an eighth and a quarter of the exponentials on the FMA pipes (816, 850: the two warps of a scheduler wait for one
// another's results longer than they gain), sixteen warps with half of the rows each (7 % slower).
constexpr int kDrawWarps = 8, kRowWarps = 4;
constexpr int kIssuer = kDrawWarps, kPlanner = kIssuer + 1, kRowFetcher = kPlanner + 1, kKeyFetcher = kRowFetcher + kRowWarps;
// Items that are known ahead.  Rows of up to two of them wait for the next ones' to be asked for before they are handed over, so the
// items behind those have to be known before they are done with.  An item without rows (a part of few) hands over what waits, so that
// is of the last two items at most, and what is drawn with is never further behind, whatever the items and however many a CTA has.
constexpr int kRing = 4;
static_assert(kRing > 2, "");
// An item's part, as every role sees it.
struct WeighUnit {
  KvSeq seq;
  long long item;    // -1: there are no more
  int head, key0, part;
  int tile0, tile1;  // row tiles
  int all_see[2];    // the first tile from which on every row sees all keys of the first 128, and of the second
  // Whether some rows of tile t are not there, or do not see all of a product's keys.
  __device__ __forceinline__ bool edge(int group, int t, int product) const {
    return t < all_see[product] || (t + 1) * kKvWeighRows > seq.rows * group;
  }
};
template <int kTiles>
__device__ __forceinline__ WeighUnit weigh_unit(const KvArrays& arrays, const WeighLists& lists, const KvWeighing& in, int heads, long long n) {
  WeighUnit u;
  u.item = n / lists.parts;
  u.part = (int)(n - u.item * lists.parts);
  int lo = 0, hi = arrays.n_seq - 1;
  while (lo < hi) {  // the last sequence that begins at or before it; ones without items share their successor's start
    const int mid = (lo + hi + 1) >> 1;
    if (lists.at[mid] * heads <= u.item) lo = mid;
    else hi = mid - 1;
  }
  const int in_head = (int)(lists.at[lo + 1] - lists.at[lo]);
  const long long rest = u.item - lists.at[lo] * heads;
  u.head = (int)(rest / in_head);
  u.key0 = (int)(rest - (long long)u.head * in_head) * 128 * kTiles;
  u.seq = arrays.seqs[lo];
  const int rows = u.seq.rows * in.group, tiles = (rows + kKvWeighRows - 1) / kKvWeighRows;
  // the first tile whose last (first) row sees `keys` keys: rows see the more the later they are
  auto first_tile = [&](int from, bool last_row, int keys) {
    int low = from, high = tiles;
    while (low < high) {
      const int mid = (low + high) >> 1, row = last_row ? min((mid + 1) * kKvWeighRows, rows) - 1 : mid * kKvWeighRows;
      if (kv_seen(u.seq.len, u.seq.rows, in.causal_block, row / in.group) >= keys) high = mid;
      else low = mid + 1;
    }
    return low;
  };
  const int seen_from = first_tile(0, true, u.key0 + 1);
  u.tile0 = seen_from + (int)((long long)(tiles - seen_from) * u.part / lists.parts);
  u.tile1 = seen_from + (int)((long long)(tiles - seen_from) * (u.part + 1) / lists.parts);
#pragma unroll
  for (int t = 0; t < 2; ++t) u.all_see[t] = t < kTiles ? first_tile(seen_from, false, u.key0 + 128 * (t + 1)) : tiles;
  return u;
}

template <int kHd, int kKind, int kTiles>
struct WeighShape {
  static constexpr int kStages = kHd == 64 ? 4 : 2;  // of Q
  static constexpr int kKeyWarps = kKind == LITEVGGT_KV_BF16 ? 1 : 2, kThreads = (kKeyFetcher + kKeyWarps) * 32;
  static constexpr int kSubBytes = 128 * 128, kTileBytes = kSubBytes * kHd / 64;
  static constexpr int kShares = kDrawWarps / (4 * kTiles);  // threads that share a key's rows
  static constexpr int kCols = 128 / kShares;                // rows of a thread in a tile
  // What is left of rows stays until they have been drawn with, Q only until it has been multiplied.  A tile's place is taken anew by the one
  // kPlaces on, whose stage is free when the product of the tile kStages before it is done; for that the draws of the tile two before
  // that one had to be over, as there are two accumulators.  kStages + 2 places do therefore.  (With Q held until it had been drawn with,
  // two sequences of 1041 rows over 10,410 keys, 16 heads of 128, took 202 us instead of 136.)
  static constexpr int kPlaces = 2 * kStages;
  static_assert(kPlaces >= kStages + 2, "");
  static constexpr int kRowInfoBytes = kPlaces * 128 * 8;
  static constexpr int kMeetBytes = (kShares - 1) * kTiles * 128 * 4;
  static constexpr int kSmemBytes = (2 * kTiles + kStages) * kTileBytes + kRowInfoBytes + kMeetBytes + 1024 + 1024;
};
template <int kStages>
struct WeighBarriers {
  WeighUnit ring[kRing];
  uint64_t unit_full[kRing], unit_empty[kRing];
  uint64_t k_full[2], k_empty[2], q_full[kStages], q_empty[kStages], d_full[2][2], d_empty[2][2], met, teardown;
  uint32_t tmem_base, abort_flag;
  int last_of_join;
};
// A row of a sequence and head, and those that follow at the same distance.
struct WeighRow {
  int row, token, head;
  __device__ __forceinline__ WeighRow(int r, int group) : row(r), token(r / group), head(r % group) {}
  __device__ __forceinline__ void advance(int rows, int tokens, int heads, int group) {  // rows = tokens * group + heads
    row += rows;
    token += tokens;
    head += heads;
    if (head >= group) head -= group, ++token;
  }
};

template <int kHd, int kKind, int kTiles>
__global__ void __launch_bounds__((WeighShape<kHd, kKind, kTiles>::kThreads), 1)
kv_weigh_tiles_kernel(const __grid_constant__ CUtensorMap k_map, KvPool pool, KvArrays arrays, KvWeighing in, WeighLists lists, long long units, uint32_t* status) {
  using Shape = WeighShape<kHd, kKind, kTiles>;
  constexpr int kKeyWarps = Shape::kKeyWarps;
  constexpr int kStages = Shape::kStages, kPlaces = Shape::kPlaces, kTileBytes = Shape::kTileBytes, kSubBytes = Shape::kSubBytes, kShares = Shape::kShares;
  constexpr int kCols = Shape::kCols, kBlock = 128 * kTiles;
  extern __shared__ uint8_t smem_raw[];
  uint8_t* smem_k = smem_raw + (-smem_u32(smem_raw) & 1023u);  // [buffer][tile] (as an offset: the compiler knows that it is shared memory)
  uint8_t* smem_q = smem_k + 2 * kTiles * kTileBytes;          // [stage]
  float* row_less = reinterpret_cast<float*>(smem_q + kStages * kTileBytes);  // [place][row]
  int* row_seen = reinterpret_cast<int*>(row_less + kPlaces * 128);           // [place][row]
  float* meet = reinterpret_cast<float*>(row_seen + kPlaces * 128);           // [share - 1][key]
  using Barriers = WeighBarriers<kStages>;
  Barriers* bars = reinterpret_cast<Barriers*>(meet + (kShares - 1) * kBlock);
  static_assert(sizeof(Barriers) <= 1024 && sizeof(WeighUnit) % 8 == 0, "");

  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  if (threadIdx.x == 0) {
    for (int i = 0; i < kRing; ++i) {
      mbar_init(&bars->unit_full[i], 1);
      mbar_init(&bars->unit_empty[i], kDrawWarps + 1 + kKeyWarps + kRowWarps);
    }
    for (int i = 0; i < 2; ++i) {
      mbar_init(&bars->k_full[i], kKeyWarps);
      mbar_init(&bars->k_empty[i], 1);
      for (int t = 0; t < 2; ++t) {
        mbar_init(&bars->d_full[t][i], 2);
        mbar_init(&bars->d_empty[t][i], kDrawWarps / kTiles);
      }
    }
    for (int i = 0; i < kStages; ++i) {
      mbar_init(&bars->q_full[i], kRowWarps);
      mbar_init(&bars->q_empty[i], 1);
    }
    mbar_init(&bars->met, kDrawWarps);
    mbar_init(&bars->teardown, 1);
    mbar_fence_init();
    bars->abort_flag = 0;
  }
  if (warp == kIssuer) {
    tmem_alloc(&bars->tmem_base, 512);
    tmem_relinquish();
  }
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tmem_base = bars->tmem_base;
  const WaitCtl ctl{&bars->abort_flag, status};
  bool ok = true;
  // The CTA's items, one after another, for every role but the planner.
  auto each_unit = [&](auto run) {
    for (uint32_t i = 0; ok; ++i) {
      ok = mbar_wait_warp(&bars->unit_full[i % kRing], (i / kRing) & 1u, ctl);
      if (!ok) break;
      const WeighUnit u = bars->ring[i % kRing];
      __syncwarp();
      if (lane == 0) mbar_arrive(&bars->unit_empty[i % kRing]);
      if (u.item < 0) break;
      run(u);
      __syncwarp();
    }
  };
  // where 16 bytes (eight channels, number `chunk`) of a tile's row lie
  auto place = [&](uint8_t* tile, int row, int chunk) { return tile + (chunk >> 3) * kSubBytes + row * 128 + ((chunk & 7) ^ (row & 7)) * 16; };

  if (warp == kPlanner) {
    // ------------------------------------------------------------------ items (a batch's arrays were there before whatever kernel is still running)
    uint32_t count = 0;
    for (long long base = blockIdx.x; ok; base += 32ll * gridDim.x) {
      const long long n = base + (long long)lane * gridDim.x;
      WeighUnit u{};
      u.item = -1;
      if (n < units) u = weigh_unit<kTiles>(arrays, lists, in, pool.kv_heads, n);
      const int there = __popc(__ballot_sync(0xffffffffu, n < units));
      for (int i = 0; i < min(there + 1, 32) && ok; ++i, ++count) {  // and behind the last one that there are no more
        ok = mbar_wait_warp(&bars->unit_empty[count % kRing], ((count / kRing) & 1u) ^ 1u, ctl);
        if (ok && lane == i) {
          bars->ring[count % kRing] = u;
          mbar_arrive(&bars->unit_full[count % kRing]);
        }
        __syncwarp();
      }
      if (there < 32) break;
    }
  } else if (kKind == LITEVGGT_KV_BF16 && warp >= kKeyFetcher) {
    // ------------------------------------------------------------------ K by TMA: lane i fetches an item's i-th page
    // (Keys behind the sequence's last page are what was there before: their scores are nobody's.)
    wait_for_previous_kernel();
    uint32_t count = 0;
    each_unit([&](const WeighUnit& u) {
      if (u.tile0 >= u.tile1) return;
      ok = mbar_wait_warp(&bars->k_empty[count & 1u], ((count >> 1) & 1u) ^ 1u, ctl);
      if (!ok) return;
      uint64_t* full = &bars->k_full[count & 1u];
      const int n = min(kBlock >> pool.page_shift, (u.seq.len - u.key0 + pool.page_size - 1) >> pool.page_shift);
      long long row = 0;
      if (lane < n) row = ((long long)arrays.pages[u.seq.page0 + (u.key0 >> pool.page_shift) + lane] * pool.kv_heads + u.head) << pool.page_shift;
      if (lane == 0) mbar_expect_tx(full, (uint32_t)(n * pool.page_size * kHd * 2));
      __syncwarp();
      if (lane < n) {
        const int at = lane << pool.page_shift;  // the page's first row of the block
        uint8_t* dst = smem_k + ((count & 1u) * kTiles + (at >> 7)) * kTileBytes + (at & 127) * 128;
#pragma unroll
        for (int s = 0; s < kHd / 64; ++s) tma_load_2d(dst + s * kSubBytes, &k_map, full, s * 64, (int)row);
      }
      __syncwarp();
      ++count;
    });
    if (lane == 0) {  // every load has landed before the CTA may go
      for (uint32_t i = 0; i < min(count, 2u); ++i) {
        const uint32_t at = count - 1 - i;
        const long long t0 = clock64();
        while (!mbar_try_wait(&bars->k_full[at & 1u], (at >> 1) & 1u)) {
          if (clock64() - t0 > kTimeoutCycles) { atomicOr(status, kStatusTimeout); break; }
        }
      }
    }
    __syncwarp();
  } else if (warp >= kKeyFetcher) {
    // ------------------------------------------------------------------ K, widened
    // Keys behind the sequence's end are zeros: their scores are nobody's, but they are scores.
    wait_for_previous_kernel();
    const int tid = threadIdx.x - kKeyFetcher * 32;
    constexpr int kThreads = kKeyWarps * 32, kRowBytes = KvRow<kHd, kKind>::kBytes, kExps = KvRow<kHd, kKind>::kExps, kPerRow = kRowBytes / 16;
    constexpr int kPasses = kBlock * kPerRow / kThreads;
    constexpr int kTogether = kPasses < 8 ? kPasses : 8;  // accesses of a thread that are under way together
    uint32_t count = 0;
    each_unit([&](const WeighUnit& u) {
      if (u.tile0 >= u.tile1) return;
      ok = mbar_wait_warp(&bars->k_empty[count & 1u], ((count >> 1) & 1u) ^ 1u, ctl);
      if (!ok) return;
      uint8_t* tiles = smem_k + (count & 1u) * kTiles * kTileBytes;
#pragma unroll 1
      for (int pass = 0; pass < kPasses; pass += kTogether) {
        uint4 x[kTogether];
        uint32_t byte[kTogether];
        int page[kTogether];
#pragma unroll
        for (int i = 0; i < kTogether; ++i) {
          const int key = u.key0 + ((pass + i) * kThreads + tid) / kPerRow;
          page[i] = key < u.seq.len ? arrays.pages[u.seq.page0 + (key >> pool.page_shift)] : 0;
        }
#pragma unroll
        for (int i = 0; i < kTogether; ++i) {
          const int piece = (pass + i) * kThreads + tid, key = u.key0 + piece / kPerRow, part = piece % kPerRow;
          const bool there = key < u.seq.len;
          const size_t row = there ? (((size_t)page[i] * pool.kv_heads + u.head) << pool.page_shift) + (key & (pool.page_size - 1)) : 0;
          const uint8_t* src = pool.k + row * kRowBytes + part * 16;
          x[i] = there ? ldg16(src) : make_uint4(0u, 0u, 0u, 0u);
          byte[i] = there ? pool.k_exp[row * kExps + (kKind == LITEVGGT_KV_E2M1 ? part : 0)] : 127u;
        }
        {
#pragma unroll
          for (int i = 0; i < kTogether; ++i) {
            const int piece = (pass + i) * kThreads + tid, row = piece / kPerRow, part = piece % kPerRow;
            uint8_t* tile = tiles + (row >> 7) * kTileBytes;
            auto put = [&](int chunk, const uint32_t* v) { *reinterpret_cast<uint4*>(place(tile, row & 127, chunk)) = make_uint4(v[0], v[1], v[2], v[3]); };
            const uint32_t w[4] = {x[i].x, x[i].y, x[i].z, x[i].w};
            if constexpr (kKind == LITEVGGT_KV_E4M3) {
              const KvFactor f = kv_factor(byte[i]);
              uint32_t v[8];
#pragma unroll
              for (int e = 0; e < 4; ++e) {
                v[2 * e] = mul_bf16x2(kv_code_bits(__byte_perm(w[e], 0u, 0x1404)), f.first * 0x10001u);
                v[2 * e + 1] = mul_bf16x2(kv_code_bits(__byte_perm(w[e], 0u, 0x3424)), f.first * 0x10001u);
              }
              if (kv_needs_second(byte[i])) {
#pragma unroll
                for (int e = 0; e < 8; ++e) v[e] = mul_bf16x2(v[e], f.second * 0x10001u);
              }
              put(2 * part, v);
              put(2 * part + 1, v + 4);
            } else {
#pragma unroll
              for (int e = 0; e < 4; ++e) {
                uint32_t v[4];
                kv4_widen(w[e], byte[i], v);
                put(4 * part + e, v);
              }
            }
          }
        }
      }
      fence_proxy_async_shared();
      __syncwarp();
      if (lane == 0) mbar_arrive(&bars->k_full[count & 1u]);
      ++count;
    });
  } else if (warp >= kRowFetcher && warp < kKeyFetcher) {
    // ------------------------------------------------------------------ Q
    // Copies of the last kLag tiles are under way, a group each; what has arrived is handed over by the threads that asked for it.
    // A thread meets every kStep-th row of a tile, eight channels of it, and kInfo rows of which it leaves what the exponentials need.
    wait_for_previous_kernel();
    const int tid = threadIdx.x - kRowFetcher * 32;
    constexpr int kThreads = kRowWarps * 32, kPerRow = kHd / 8, kStep = kThreads / kPerRow, kInfo = 128 / kThreads;
    constexpr uint32_t kLag = kStages > 2 ? 2 : 1;
    const int group = in.group, step_tokens = kStep / group, step_heads = kStep % group, info_tokens = kThreads / group, info_heads = kThreads % group;
    const uint32_t row_stride = (uint32_t)in.q_stride.row, head_stride = (uint32_t)in.q_stride.head;  // (elements; less than 2^32)
    uint32_t count = 0, given = 0;
    auto hand_over = [&]() {  // the oldest, which has arrived
      fence_proxy_async_shared();
      __syncwarp();
      if (lane == 0) mbar_arrive(&bars->q_full[given % kStages]);
      ++given;
    };
    each_unit([&](const WeighUnit& u) {
      if (u.tile0 >= u.tile1) {  // nothing of this item drives on what is under way, and the next item may never be known without that
        cp_async_wait<0>();
        while (given != count) hand_over();
        return;
      }
      const int rows = u.seq.rows * group;
      WeighRow mine(u.tile0 * kKvWeighRows + tid / kPerRow, group), info(u.tile0 * kKvWeighRows + tid, group);
      float ahead[kInfo];  // the next tile's
      auto look_ahead = [&]() {
        WeighRow r = info;
#pragma unroll
        for (int i = 0; i < kInfo; ++i) {
          ahead[i] = r.row < rows ? in.lse[(long long)(u.seq.row0 + r.token) * in.q_heads + u.head * group + r.head] : 0.0f;
          r.advance(kThreads, info_tokens, info_heads, group);
        }
      };
      look_ahead();
      for (int t = u.tile0; t < u.tile1; ++t) {
        const uint32_t stage = count % kStages;
        const bool edge = u.edge(group, t, kTiles - 1);  // (of the first keys only where of the last)
        float less[kInfo];
        int seen[kInfo];
#pragma unroll
        for (int i = 0; i < kInfo; ++i) {
          less[i] = ahead[i];
          seen[i] = edge && info.row < rows ? kv_seen(u.seq.len, u.seq.rows, in.causal_block, info.token) : 0;  // (looked at where there is an edge)
          info.advance(kThreads, info_tokens, info_heads, group);
        }
        if (t + 1 < u.tile1) look_ahead();
        ok = mbar_wait_warp(&bars->q_empty[stage], ((count / kStages) & 1u) ^ 1u, ctl);
        if (!ok) return;
        const uint32_t place_of_tile = count % kPlaces;
        ++count;
        uint8_t* tile = smem_q + stage * kTileBytes;
#pragma unroll
        for (int i = 0; i < 128 / kStep; ++i) {
          const bool there = mine.row < rows;
          const unsigned long long at = (unsigned long long)(uint32_t)(u.seq.row0 + mine.token) * row_stride +
                                        (unsigned long long)(uint32_t)(u.head * group + mine.head) * head_stride;
          cp_async16(place(tile, tid / kPerRow + i * kStep, tid % kPerRow), in.q + (there ? at : 0) + (tid % kPerRow) * 8, there);
          mine.advance(kStep, step_tokens, step_heads, group);
        }
        cp_async_commit();
#pragma unroll
        for (int i = 0; i < kInfo; ++i) {
          row_less[place_of_tile * 128 + i * kThreads + tid] = -kLog2e * less[i];
          row_seen[place_of_tile * 128 + i * kThreads + tid] = seen[i];
        }
        if (count - given > kLag) {
          cp_async_wait<kLag>();
          hand_over();
        }
      }
    });
    cp_async_wait<0>();  // every copy has landed before the CTA may go
    while (ok && given != count) hand_over();
  } else if (warp == kIssuer) {
    // ------------------------------------------------------------------ products: one lane
    constexpr uint32_t idesc = umma_idesc_bf16(128, 128, false, false);
    const uint64_t k_desc0 = smem_desc_sw128(smem_u32(smem_k), 16, 1024), q_desc0 = smem_desc_sw128(smem_u32(smem_q), 16, 1024);
    uint32_t k_count = 0, q_count = 0;
    bool issued = true;  // (the issuing lane's: all of it went well)
    each_unit([&](const WeighUnit& u) {
      if (elect_one() && u.tile0 < u.tile1) {  // the same lane every time
        const uint32_t buffer = k_count & 1u;
        issued = issued && mbar_wait(&bars->k_full[buffer], (k_count >> 1) & 1u, ctl);
        for (int t = u.tile0; t < u.tile1 && issued; ++t, ++q_count) {
          const uint32_t stage = q_count % kStages, slot = q_count & 1u;
          issued = mbar_wait(&bars->q_full[stage], (q_count / kStages) & 1u, ctl);
#pragma unroll
          for (int kt = 0; kt < kTiles; ++kt) {
            issued = issued && mbar_wait(&bars->d_empty[kt][slot], ((q_count >> 1) & 1u) ^ 1u, ctl);
            if (!issued) break;
            tc_fence_after();
#pragma unroll
            for (int k = 0; k < kHd / 16; ++k) {
              const uint64_t in_tile = (uint64_t)(((k >> 2) * kSubBytes + (k & 3) * 32) >> 4);
              umma_ss(tmem_base + (kt * 2 + slot) * 128, k_desc0 + (uint64_t)(((buffer * kTiles + kt) * kTileBytes) >> 4) + in_tile,
                      q_desc0 + (uint64_t)((stage * kTileBytes) >> 4) + in_tile, idesc, k != 0 ? 1u : 0u);
            }
            umma_commit(&bars->d_full[kt][slot]);
            mbar_arrive(&bars->d_full[kt][slot]);  // (and with it what the fetchers have left in shared memory)
          }
          if (issued) umma_commit(&bars->q_empty[stage]);
        }
        if (issued) umma_commit(&bars->k_empty[buffer]);
        ++k_count;
      }
      __syncwarp();
    });
    if (elect_one() && !(issued && ok)) {  // what is under way must have retired before tensor memory is given up
      umma_commit(&bars->teardown);
      const long long t0 = clock64();
      while (!mbar_try_wait(&bars->teardown, 0)) {
        if (clock64() - t0 > kTimeoutCycles) break;
      }
    }
    __syncwarp();
  } else {
    // ------------------------------------------------------------------ exponentials: a thread is a key against a share of the rows
    wait_for_previous_kernel();
    const int kt = warp / (4 * kShares), share = (warp >> 2) % kShares, key_in = kt * 128 + (warp & 3) * 32 + lane;
    const uint32_t d_addr = tmem_base + ((uint32_t)((warp & 3) * 32) << 16) + kt * 256 + share * kCols;
    uint32_t count = 0, meetings = 0;
    auto all_draw = [&]() {  // the eight warps; bounded like every wait
      __syncwarp();
      if (lane == 0) mbar_arrive(&bars->met);
      ok = mbar_wait_warp(&bars->met, meetings & 1u, ctl) && ok;
      ++meetings;
    };
    const float2 scale2 = make_float2(in.scale_log2, in.scale_log2);
    each_unit([&](const WeighUnit& u) {
      const int key = u.key0 + key_in;
      float total = 0.0f, some = 0.0f;
      for (int t = u.tile0; t < u.tile1; ++t, ++count) {
        const uint32_t place_of_tile = count % kPlaces, slot = count & 1u;
        ok = mbar_wait_warp(&bars->d_full[kt][slot], (count >> 1) & 1u, ctl);
        if (!ok) return;
        tc_fence_after();
        const float* less = row_less + place_of_tile * 128 + share * kCols;
        const int* seen = row_seen + place_of_tile * 128 + share * kCols;
        auto tile_sum = [&](auto edge_constant) {
          constexpr bool kEdge = decltype(edge_constant)::value;
          float2 sum[2] = {make_float2(0.0f, 0.0f), make_float2(0.0f, 0.0f)};
          uint32_t x[2][32];  // the next 32 are on their way while these are worked on
          tmem_ld32(d_addr + slot * 128, x[0]);
#pragma unroll
          for (int c = 0; c < kCols / 32; ++c) {
            tmem_ld_wait();
            if (c + 1 < kCols / 32) tmem_ld32(d_addr + slot * 128 + (c + 1) * 32, x[(c + 1) & 1]);
            const uint32_t (&now)[32] = x[c & 1];
#pragma unroll
            for (int i = 0; i < 16; ++i) {
              const float4 l4 = *reinterpret_cast<const float4*>(less + c * 32 + (2 * i & ~3));
              const float2 l = i & 1 ? make_float2(l4.z, l4.w) : make_float2(l4.x, l4.y);
              float2 y = __ffma2_rn(make_float2(__uint_as_float(now[2 * i]), __uint_as_float(now[2 * i + 1])), scale2, l);
              y = make_float2(fast_exp2(y.x), fast_exp2(y.y));
              if constexpr (kEdge) {
                const int2 s = *reinterpret_cast<const int2*>(seen + c * 32 + 2 * i);
                y = make_float2(key < s.x ? y.x : 0.0f, key < s.y ? y.y : 0.0f);
              }
              sum[i & 1] = __fadd2_rn(sum[i & 1], y);
            }
          }
          sum[0] = __fadd2_rn(sum[0], sum[1]);
          return sum[0].x + sum[0].y;
        };
        const float sum = u.edge(in.group, t, kt) ? tile_sum(std::true_type{}) : tile_sum(std::false_type{});
        tc_fence_before();
        __syncwarp();
        if (lane == 0) mbar_arrive(&bars->d_empty[kt][slot]);
        // A tile's own sum first, 32 tiles' next, and those one after another: rows are added in chains of 32, 32 and one for every 4,096
        // of them.  (Tile after tile, 256,000 rows that give alike are off by up to 2^-15.)
        some += sum;
        if (((t - u.tile0) & 31) == 31) total += some, some = 0.0f;
      }
      total += some;
      // the threads of a key, in their order
      if constexpr (kShares > 1) {
        if (share > 0) meet[(share - 1) * kBlock + key_in] = total;
        all_draw();
#pragma unroll
        for (int i = 1; i < kShares; ++i) total += meet[(i - 1) * kBlock + key_in];  // (of the first share)
      }
      bool mine = share == 0 && key < u.seq.len;
      if (lists.parts > 1) {  // whoever comes last adds the parts up, in their order
        float* parts = lists.sums + u.item * lists.parts * kBlock + key_in;
        if (share == 0) __stcg(parts + (long long)u.part * kBlock, total);
        __threadfence();
        all_draw();
        if (threadIdx.x == 0) {
          const int last = atomicAdd(lists.joins + u.item, 1) == lists.parts - 1 ? 1 : 0;
          if (last) lists.joins[u.item] = 0;
          *reinterpret_cast<volatile int*>(&bars->last_of_join) = last;
        }
        all_draw();
        mine = mine && *reinterpret_cast<volatile int*>(&bars->last_of_join) != 0;
        if (mine) {
          __threadfence();
          total = 0.0f;
          for (int p = 0; p < lists.parts; ++p) total += __ldcg(parts + (long long)p * kBlock);
        }
      }
      if (mine && ok) {
        const size_t page = (size_t)arrays.pages[u.seq.page0 + (key >> pool.page_shift)];
        float* w = pool.weights + ((page * pool.kv_heads + u.head) << pool.page_shift) + (key & (pool.page_size - 1));
        *w = tallied(in.decay, in.decay == 0.0f ? 0.0f : *w, total);
      }
      if (kShares > 1) all_draw();  // what was met with may be written again
    });
  }
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  if (warp == kIssuer) tmem_dealloc(tmem_base, 512);
}

template <int kHd, int kKind, int kTiles>
cudaError_t start_tiles(const litevggt_kv_cache& c, const litevggt_kv_batch& b, const KvWeighing& w, cudaStream_t s) {
  using Shape = WeighShape<kHd, kKind, kTiles>;
  static_assert(Shape::kSmemBytes <= 227 * 1024, "");
  auto kernel = kv_weigh_tiles_kernel<kHd, kKind, kTiles>;
  static std::atomic<unsigned long long> done{0};
  const cudaError_t e = set_max_dynamic_smem_once(reinterpret_cast<const void*>(kernel), Shape::kSmemBytes, done);
  if (e != cudaSuccess) return e;
  const WeighLists lists{reinterpret_cast<const long long*>(b.base + b.o_tiles_at), b.weigh.parts, reinterpret_cast<int*>(b.base + b.o_weigh_joins),
                         reinterpret_cast<float*>(b.base + b.o_weigh_sums)};
  const long long units = b.weigh.items * b.weigh.parts;
  return launch(kernel, dim3((unsigned)std::min(units, (long long)c.num_sms)), (unsigned)Shape::kThreads, (size_t)Shape::kSmemBytes, s, c.k_map, c.pool, kv_arrays(b), w, lists,
                units, c.status);
}

template <class F>
cudaError_t by_kind(const litevggt_kv_cache& c, const F& f) {
  using std::integral_constant;
  auto kinds = [&](auto hd) {
    if (c.cfg.dtype == LITEVGGT_KV_E2M1) return f(hd, integral_constant<int, LITEVGGT_KV_E2M1>{});
    if (c.cfg.dtype == LITEVGGT_KV_E4M3) return f(hd, integral_constant<int, LITEVGGT_KV_E4M3>{});
    return f(hd, integral_constant<int, LITEVGGT_KV_BF16>{});
  };
  return c.cfg.head_dim == 64 ? kinds(integral_constant<int, 64>{}) : kinds(integral_constant<int, 128>{});
}

}  // namespace

cudaError_t launch_kv_weigh_few(const litevggt_kv_cache& c, const litevggt_kv_batch& b, const KvWeighing& w, cudaStream_t s, int* launches) {
  const long long units = b.weigh.few_at.back() * c.cfg.kv_heads;
  if (units == 0) return cudaSuccess;
  const WeighLists lists{reinterpret_cast<const long long*>(b.base + b.o_few_at), 1, nullptr, nullptr};
  ++*launches;
  return by_kind(c, [&](auto hd, auto kind) {
    constexpr int kHd = decltype(hd)::value, kKind = decltype(kind)::value;
    // A warp's run: as short as the chip allows, but no shorter than a unit.
    const long long warps = std::min(units, (long long)c.num_sms * FewKeys<kHd, kKind>::kBlocks * kWeighWarps), per_warp = (units + warps - 1) / warps;
    const unsigned blocks = (unsigned)(((units + per_warp - 1) / per_warp + kWeighWarps - 1) / kWeighWarps);
    auto go = [&](auto kernel) { return launch(kernel, dim3(blocks), kWeighWarps * 32, 0, s, c.pool, kv_arrays(b), w, lists, per_warp, units); };
    return b.few_rows <= 8 ? go(kv_weigh_few_kernel<kHd, kKind, true>) : go(kv_weigh_few_kernel<kHd, kKind, false>);
  });
}

cudaError_t launch_kv_weigh_tiles(const litevggt_kv_cache& c, const litevggt_kv_batch& b, const KvWeighing& w, cudaStream_t s, int* launches) {
  if (b.weigh.items == 0) return cudaSuccess;
  ++*launches;
  return by_kind(c, [&](auto hd, auto kind) {
    constexpr int kHd = decltype(hd)::value, kKind = decltype(kind)::value;
    return b.weigh.key_block == 256 ? start_tiles<kHd, kKind, 2>(c, b, w, s) : start_tiles<kHd, kKind, 1>(c, b, w, s);
  });
}

}  // namespace lv
