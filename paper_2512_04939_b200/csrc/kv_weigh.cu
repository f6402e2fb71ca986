// What cached tokens draw of the attention of a batch's rows, given each row's log-sum-exp:
//   w_j = decay w_j + sum_i p_ij,   p_ij = 2^(c q_i k_j - l_i)  for the rows i that see the key j
// Nothing is multiplied by V, and a key's sum runs over rows, so the scores are taken with keys as the product's rows: a thread owns a
// key, adds along its own row and needs nobody else's numbers.  What a row does not see is left out by a comparison, so nothing that
// lies there has any influence.
#include "exp2.cuh"
#include "kv_cache.h"
#include "kv_mma.cuh"
#include "kv_quant.cuh"

namespace lv {

namespace {

constexpr float kLog2e = 1.4426950408889634f;

// What a launch over either kind of sequence is given.
struct WeighLists {
  const long long* at;  // units or items of a head before each sequence
  int parts;
  int* joins;
  float* sums;
};

// The sequence that number n of all heads' units belongs to.
__device__ __forceinline__ int seq_of_unit(const long long* at, int n_seq, int heads, long long n) {
  int lo = 0, hi = n_seq - 1;
  while (lo < hi) {  // the last one that begins at or before it; ones without units share their successor's start
    const int mid = (lo + hi + 1) >> 1;
    if (at[mid] * heads <= n) lo = mid;
    else hi = mid - 1;
  }
  return lo;
}

__device__ __forceinline__ float tallied(float decay, float before, float sum) { return decay == 0.0f ? sum : fmaf(decay, before, sum); }

// ------------------------------------------------------------------ few rows
// A warp's unit is 32 keys of a head, whose K rows it loads straight into the fragments of mma.m16n8k16 with Q as the other operand:
// the four lanes of a key read its row in 16 bytes each (or a quarter row each), and the contraction runs over the channels in that order.
// HBM bounds it: K once, 4 operations a byte at one row; a unit's 4 KB are all under way at once.
constexpr int kWeighWarps = 4;

template <int kHd, int kKind, bool kHalf>
struct FewKeys {
  static constexpr int kRowBytes = KvRow<kHd, kKind>::kBytes, kExps = KvRow<kHd, kKind>::kExps;
  static constexpr int kRun = kKind == LITEVGGT_KV_BF16 ? 8 : kKind == LITEVGGT_KV_E4M3 ? 16 : kHd / 4;  // channels side by side in a lane
  static constexpr int kWords = kRowBytes / 16;  // of a lane: a quarter of the row
  uint32_t w[4][kWords];                         // of the keys lane / 4 of four tiles of 8
  uint32_t byte[4];
};

template <int kHd, int kKind, bool kHalf>
__global__ void __launch_bounds__(kWeighWarps * 32)
kv_weigh_few_kernel(KvPool pool, KvArrays arrays, KvWeighing in, WeighLists lists, long long per_warp, long long units) {
  using Keys = FewKeys<kHd, kKind, kHalf>;
  constexpr int kHalves = kHalf ? 1 : 2, kRun = Keys::kRun, kSteps = kHd / 16;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, g = lane >> 2, q4 = lane & 3;
  long long unit = ((long long)blockIdx.x * kWeighWarps + warp) * per_warp;
  const long long end = min(unit + per_warp, units);
  wait_for_previous_kernel();
  if (unit >= end) return;
  int s = seq_of_unit(lists.at, arrays.n_seq, pool.kv_heads, unit);
  long long in_head = lists.at[s + 1] - lists.at[s];
  const long long rest = unit - lists.at[s] * pool.kv_heads;
  int head = (int)(rest / in_head), key0 = (int)(rest % in_head) * kKvWeighUnit;
  KvSeq seq = arrays.seqs[s];
  bool fresh = true;

  uint32_t qa[kSteps][2 * kHalves];
  float less[kHalves];  // the rows' log-sum-exp in base 2
  int seen[kHalves];
  for (; unit < end; ++unit) {
    Keys k;
    size_t row0[2];  // of the pool, of each 16 keys
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      const int key = min(key0 + 16 * h, seq.len - 1) & ~15;  // (of a second half that is not there the first's rows)
      const size_t page = (size_t)arrays.pages[seq.page0 + (key >> pool.page_shift)];
      row0[h] = ((page * pool.kv_heads + head) << pool.page_shift) + (key & (pool.page_size - 1));
    }
#pragma unroll
    for (int t = 0; t < 4; ++t) {
      const size_t row = row0[t >> 1] + 8 * (t & 1) + g;
      const uint8_t* src = pool.k + row * Keys::kRowBytes;
      if constexpr (Keys::kWords == 2) {
        const uint2 x = *reinterpret_cast<const uint2*>(src + q4 * 8);
        k.w[t][0] = x.x, k.w[t][1] = x.y;
      } else {
#pragma unroll
        for (int i = 0; i < Keys::kWords / 4; ++i) {
          const uint4 x = ldg16(src + (i * 4 + q4) * 16);
          k.w[t][4 * i] = x.x, k.w[t][4 * i + 1] = x.y, k.w[t][4 * i + 2] = x.z, k.w[t][4 * i + 3] = x.w;
        }
      }
      if constexpr (Keys::kExps > 0) k.byte[t] = pool.k_exp[row * Keys::kExps + (kKind == LITEVGGT_KV_E2M1 ? q4 * Keys::kExps / 4 : 0)];
    }
    if (fresh) {  // the rows
      fresh = false;
      const int rows = seq.rows * in.group;
#pragma unroll
      for (int half = 0; half < kHalves; ++half) {
        const int r = g + 8 * half;
        const bool live = r < rows;
        const int token = live ? r / in.group : 0, q_head = head * in.group + (live ? r % in.group : 0);
        const __nv_bfloat16* src = in.q + (seq.row0 + token) * in.q_stride.row + q_head * in.q_stride.head;
#pragma unroll
        for (int i = 0; i < kHd / (4 * kRun); ++i)
#pragma unroll
          for (int j = 0; j < kRun / 4; ++j) {
            const uint2 x = live ? *reinterpret_cast<const uint2*>(src + (i * 4 + q4) * kRun + 4 * j) : make_uint2(0u, 0u);
            qa[i * (kRun / 4) + j][half] = x.x;
            qa[i * (kRun / 4) + j][kHalves + half] = x.y;
          }
        less[half] = live ? -kLog2e * in.lse[(long long)(seq.row0 + token) * in.q_heads + q_head] : 0.0f;
        seen[half] = live ? kv_seen(seq.len, seq.rows, in.causal_block, token) : 0;
      }
    }
    float drawn[4][2];  // of the keys 2 q4 and 2 q4 + 1 of each tile, over this lane's rows
#pragma unroll
    for (int t = 0; t < 4; ++t) {
      float c[4] = {0.0f, 0.0f, 0.0f, 0.0f};
      auto step = [&](int n, uint32_t b0, uint32_t b1) {
        if constexpr (kHalf) mma_16816<false>(c, qa[n][0], 0u, qa[n][1], 0u, b0, b1);
        else mma_16816<false>(c, qa[n][0], qa[n][kHalves - 1], qa[n][kHalves], qa[n][2 * kHalves - 1], b0, b1);
      };
      if constexpr (kKind == LITEVGGT_KV_BF16) {
#pragma unroll
        for (int n = 0; n < kSteps; ++n) step(n, k.w[t][2 * n], k.w[t][2 * n + 1]);
      } else if constexpr (kKind == LITEVGGT_KV_E4M3) {
        const KvFactor f = kv_factor(k.byte[t]);
#pragma unroll
        for (int n = 0; n < kSteps; ++n) {
          uint32_t lo = mul_bf16x2(kv_code_bits(__byte_perm(k.w[t][n], 0u, 0x1404)), f.first * 0x10001u);
          uint32_t hi = mul_bf16x2(kv_code_bits(__byte_perm(k.w[t][n], 0u, 0x3424)), f.first * 0x10001u);
          if (kv_needs_second(k.byte[t])) lo = mul_bf16x2(lo, f.second * 0x10001u), hi = mul_bf16x2(hi, f.second * 0x10001u);
          step(n, lo, hi);
        }
      } else {
#pragma unroll
        for (int i = 0; i < kHd / 32; ++i) {
          uint32_t x[4];
          kv4_widen(k.w[t][i], k.byte[t], x);
          step(2 * i, x[0], x[1]);
          step(2 * i + 1, x[2], x[3]);
        }
      }
#pragma unroll
      for (int e = 0; e < 2; ++e) {
        const int key = key0 + 8 * t + 2 * q4 + e;
        drawn[t][e] = 0.0f;
#pragma unroll
        for (int half = 0; half < kHalves; ++half) {
          const float p = fast_exp2(fmaf(c[2 * half + e], in.scale_log2, less[half]));
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
    if (key0 + 16 * (upper ? 1 : 0) + in16 < seq.len) {
      float* w = pool.weights + (upper ? row0[1] : row0[0]) + in16;
      *w = tallied(in.decay, in.decay == 0.0f ? 0.0f : *w, sum);
    }
    // the next unit: the next keys, the next head, or the next sequence that has units
    key0 += kKvWeighUnit;
    if (key0 >= seq.len) {
      key0 = 0;
      fresh = true;
      if (++head == pool.kv_heads && unit + 1 < end) {
        head = 0;
        do ++s;
        while (lists.at[s + 1] == lists.at[s]);
        seq = arrays.seqs[s];
      }
    }
  }
}

// ------------------------------------------------------------------ chunks
// Scores on the 5th-generation tensor cores, 128 keys by 128 rows a product, kTiles of them side by side against the same rows.  One
// exponential a score and 64 (128) multiplications for it, so the special-function unit is the bound, at 16 a clock; the products need
// an eighth (a quarter) of its time.  Roles: 16 warps take the exponentials, each thread a key against a share of the rows; one issues the
// products; four fetch K once an item and Q tile by tile into swizzled shared memory (widening codes on the way), with what the
// exponentials need of a row: its log-sum-exp and how many keys it sees.
constexpr int kDrawWarps = 16, kFetchWarps = 4, kWeighThreads = (kDrawWarps + 1 + kFetchWarps) * 32;

template <int kHd, int kTiles>
struct WeighShape {
  static constexpr int kStages = kHd == 64 ? 4 : 2;  // of Q
  static constexpr int kSubBytes = 128 * 128, kTileBytes = kSubBytes * kHd / 64;
  static constexpr int kShares = 4 / kTiles;         // threads that share a key's rows
  static constexpr int kCols = 128 / kShares;        // rows of a thread in a tile
  static constexpr int kRowInfoBytes = kStages * 128 * 8;
  static constexpr int kMeetBytes = (kShares - 1) * kTiles * 128 * 4;
  static constexpr int kSmemBytes = (2 * kTiles + kStages) * kTileBytes + kRowInfoBytes + kMeetBytes + 512 + 1024;
};
template <int kStages>
struct WeighBarriers {
  uint64_t k_full[2], k_empty[2], q_full[kStages], q_empty[kStages], d_full[2][2], d_empty[2][2], teardown;
  uint32_t tmem_base, abort_flag;
  int last_of_join;
};

// An item's part, as every role sees it.
struct WeighUnit {
  KvSeq seq;
  long long item;
  int head, key0, part;
  int tile0, tile1;  // row tiles
};
template <int kBlock>
__device__ __forceinline__ WeighUnit weigh_unit(const KvArrays& arrays, const WeighLists& lists, const KvWeighing& in, int heads, long long n) {
  WeighUnit u;
  u.item = n / lists.parts;
  u.part = (int)(n % lists.parts);
  const int s = seq_of_unit(lists.at, arrays.n_seq, heads, u.item);
  const long long in_head = lists.at[s + 1] - lists.at[s], rest = u.item - lists.at[s] * heads;
  u.head = (int)(rest / in_head);
  u.key0 = (int)(rest % in_head) * kBlock;
  u.seq = arrays.seqs[s];
  const int rows = u.seq.rows * in.group, tiles = (rows + kKvWeighRows - 1) / kKvWeighRows;
  // the first tile of which a row sees the first key: rows see the more the later they are
  int lo = 0, hi = tiles;
  while (lo < hi) {
    const int mid = (lo + hi) >> 1, last = min((mid + 1) * kKvWeighRows, rows) - 1;
    if (kv_seen(u.seq.len, u.seq.rows, in.causal_block, last / in.group) > u.key0) hi = mid;
    else lo = mid + 1;
  }
  u.tile0 = lo + (int)((long long)(tiles - lo) * u.part / lists.parts);
  u.tile1 = lo + (int)((long long)(tiles - lo) * (u.part + 1) / lists.parts);
  return u;
}

template <int kHd, int kKind, int kTiles>
__global__ void __launch_bounds__(kWeighThreads, 1)
kv_weigh_tiles_kernel(KvPool pool, KvArrays arrays, KvWeighing in, WeighLists lists, long long units, uint32_t* status) {
  using Shape = WeighShape<kHd, kTiles>;
  constexpr int kStages = Shape::kStages, kTileBytes = Shape::kTileBytes, kSubBytes = Shape::kSubBytes, kShares = Shape::kShares;
  constexpr int kCols = Shape::kCols, kBlock = 128 * kTiles;
  extern __shared__ uint8_t smem_raw[];
  uint8_t* smem_k = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~uintptr_t(1023));  // [buffer][tile]
  uint8_t* smem_q = smem_k + 2 * kTiles * kTileBytes;                                                              // [stage]
  float* row_less = reinterpret_cast<float*>(smem_q + kStages * kTileBytes);                                       // [stage][row]
  int* row_seen = reinterpret_cast<int*>(row_less + kStages * 128);                                                // [stage][row]
  float* meet = reinterpret_cast<float*>(row_seen + kStages * 128);                                                // [share - 1][key]
  using Barriers = WeighBarriers<kStages>;
  Barriers* bars = reinterpret_cast<Barriers*>(meet + (kShares - 1) * kBlock);
  static_assert(sizeof(Barriers) <= 512, "");

  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  constexpr int kIssuer = kDrawWarps, kFetcher = kIssuer + 1;
  if (threadIdx.x == 0) {
    for (int i = 0; i < 2; ++i) {
      mbar_init(&bars->k_full[i], kFetchWarps);
      mbar_init(&bars->k_empty[i], 1);
      for (int t = 0; t < 2; ++t) {
        mbar_init(&bars->d_full[t][i], 1);
        mbar_init(&bars->d_empty[t][i], kDrawWarps / kTiles);
      }
    }
    for (int i = 0; i < kStages; ++i) {
      mbar_init(&bars->q_full[i], kFetchWarps);
      mbar_init(&bars->q_empty[i], 1 + kDrawWarps);
    }
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
  wait_for_previous_kernel();
  auto unit_of = [&](long long n) { return weigh_unit<kBlock>(arrays, lists, in, pool.kv_heads, n); };

  if (warp >= kFetcher) {
    // ------------------------------------------------------------------ K and Q
    const int tid = threadIdx.x - kFetcher * 32;
    constexpr int kThreads = kFetchWarps * 32, kAhead = 8;  // accesses of a thread that are under way together
    bool ok = true;
    uint32_t k_count = 0, q_count = 0;
    auto given = [&](uint64_t* bar) {
      fence_proxy_async_shared();
      __syncwarp();
      if (lane == 0) mbar_arrive(bar);
    };
    // where 16 bytes (eight channels, number `chunk`) of a tile's row lie
    auto place = [&](uint8_t* tile, int row, int chunk) {
      return reinterpret_cast<uint4*>(tile + (chunk >> 3) * kSubBytes + row * 128 + ((chunk & 7) ^ (row & 7)) * 16);
    };
    for (long long n = blockIdx.x; n < units && ok; n += gridDim.x) {
      const WeighUnit u = unit_of(n);
      if (u.tile0 >= u.tile1) continue;
      const uint32_t buffer = k_count & 1u;
      ok = mbar_wait_warp(&bars->k_empty[buffer], ((k_count >> 1) & 1u) ^ 1u, ctl);
      if (!ok) break;
      {  // keys behind the sequence's end are zeros: their scores are nobody's, but they are scores
        constexpr int kRowBytes = KvRow<kHd, kKind>::kBytes, kExps = KvRow<kHd, kKind>::kExps, kPerRow = kRowBytes / 16;
        constexpr int kPasses = kBlock * kPerRow / kThreads, kTogether = kPasses < kAhead ? kPasses : kAhead;
        uint8_t* tiles = smem_k + buffer * kTiles * kTileBytes;
#pragma unroll 1
        for (int pass = 0; pass < kPasses; pass += kTogether) {
          uint4 x[kTogether];
          uint32_t byte[kTogether];
#pragma unroll
          for (int i = 0; i < kTogether; ++i) {
            const int piece = (pass + i) * kThreads + tid, key = u.key0 + piece / kPerRow, part = piece % kPerRow;
            x[i] = make_uint4(0u, 0u, 0u, 0u);
            byte[i] = 127u;
            if (key < u.seq.len) {
              const size_t page = (size_t)arrays.pages[u.seq.page0 + (key >> pool.page_shift)];
              const size_t row = ((page * pool.kv_heads + u.head) << pool.page_shift) + (key & (pool.page_size - 1));
              x[i] = ldg16(pool.k + row * kRowBytes + part * 16);
              if constexpr (kExps > 0) byte[i] = pool.k_exp[row * kExps + (kKind == LITEVGGT_KV_E2M1 ? part : 0)];
            }
          }
#pragma unroll
          for (int i = 0; i < kTogether; ++i) {
            const int piece = (pass + i) * kThreads + tid, row = piece / kPerRow, part = piece % kPerRow;
            uint8_t* tile = tiles + (row >> 7) * kTileBytes;
            const uint32_t w[4] = {x[i].x, x[i].y, x[i].z, x[i].w};
            if constexpr (kKind == LITEVGGT_KV_BF16) {
              *place(tile, row & 127, part) = x[i];
            } else if constexpr (kKind == LITEVGGT_KV_E4M3) {
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
              *place(tile, row & 127, 2 * part) = make_uint4(v[0], v[1], v[2], v[3]);
              *place(tile, row & 127, 2 * part + 1) = make_uint4(v[4], v[5], v[6], v[7]);
            } else {
#pragma unroll
              for (int e = 0; e < 4; ++e) {
                uint32_t v[4];
                kv4_widen(w[e], byte[i], v);
                *place(tile, row & 127, 4 * part + e) = make_uint4(v[0], v[1], v[2], v[3]);
              }
            }
          }
        }
      }
      given(&bars->k_full[buffer]);
      ++k_count;
      const int rows = u.seq.rows * in.group;
      for (int t = u.tile0; t < u.tile1; ++t, ++q_count) {
        const uint32_t stage = q_count % kStages;
        ok = mbar_wait_warp(&bars->q_empty[stage], ((q_count / kStages) & 1u) ^ 1u, ctl);
        if (!ok) break;
        constexpr int kPerRow = kHd / 8, kPasses = 128 * kPerRow / kThreads, kTogether = kPasses < kAhead ? kPasses : kAhead;
        uint8_t* tile = smem_q + stage * kTileBytes;
        const int base = t * kKvWeighRows;
        {  // this thread's row
          const int r = base + tid;
          const bool live = r < rows;
          const int token = live ? r / in.group : 0, q_head = u.head * in.group + (live ? r % in.group : 0);
          row_less[stage * 128 + tid] = live ? -kLog2e * in.lse[(long long)(u.seq.row0 + token) * in.q_heads + q_head] : 0.0f;
          row_seen[stage * 128 + tid] = live ? kv_seen(u.seq.len, u.seq.rows, in.causal_block, token) : 0;
        }
#pragma unroll 1
        for (int pass = 0; pass < kPasses; pass += kTogether) {
          uint4 x[kTogether];
#pragma unroll
          for (int i = 0; i < kTogether; ++i) {
            const int piece = (pass + i) * kThreads + tid, r = base + piece / kPerRow, part = piece % kPerRow;
            x[i] = make_uint4(0u, 0u, 0u, 0u);
            if (r < rows) {
              const int token = r / in.group, q_head = u.head * in.group + r % in.group;
              x[i] = ldg16(in.q + (u.seq.row0 + token) * in.q_stride.row + q_head * in.q_stride.head + part * 8);
            }
          }
#pragma unroll
          for (int i = 0; i < kTogether; ++i) {
            const int piece = (pass + i) * kThreads + tid;
            *place(tile, piece / kPerRow, piece % kPerRow) = x[i];
          }
        }
        given(&bars->q_full[stage]);
      }
    }
  } else if (warp == kIssuer) {
    // ------------------------------------------------------------------ products: one lane
    bool ok = true;
    if (elect_one()) {
      constexpr uint32_t idesc = umma_idesc_bf16(128, 128, false, false);
      const uint64_t k_desc0 = smem_desc_sw128(smem_u32(smem_k), 16, 1024), q_desc0 = smem_desc_sw128(smem_u32(smem_q), 16, 1024);
      uint32_t k_count = 0, q_count = 0;
      for (long long n = blockIdx.x; n < units && ok; n += gridDim.x) {
        const WeighUnit u = unit_of(n);
        if (u.tile0 >= u.tile1) continue;
        const uint32_t buffer = k_count & 1u;
        ok = mbar_wait(&bars->k_full[buffer], (k_count >> 1) & 1u, ctl);
        for (int t = u.tile0; t < u.tile1 && ok; ++t, ++q_count) {
          const uint32_t stage = q_count % kStages, slot = q_count & 1u;
          ok = mbar_wait(&bars->q_full[stage], (q_count / kStages) & 1u, ctl);
#pragma unroll
          for (int kt = 0; kt < kTiles; ++kt) {
            ok = ok && mbar_wait(&bars->d_empty[kt][slot], ((q_count >> 1) & 1u) ^ 1u, ctl);
            if (!ok) break;
            tc_fence_after();
#pragma unroll
            for (int k = 0; k < kHd / 16; ++k) {
              const uint64_t in_tile = (uint64_t)(((k >> 2) * kSubBytes + (k & 3) * 32) >> 4);
              umma_ss(tmem_base + (kt * 2 + slot) * 128, k_desc0 + (uint64_t)(((buffer * kTiles + kt) * kTileBytes) >> 4) + in_tile,
                      q_desc0 + (uint64_t)((stage * kTileBytes) >> 4) + in_tile, idesc, k != 0 ? 1u : 0u);
            }
            umma_commit(&bars->d_full[kt][slot]);
          }
          if (ok) umma_commit(&bars->q_empty[stage]);
        }
        if (ok) umma_commit(&bars->k_empty[buffer]);
        ++k_count;
      }
      if (!ok) {  // what is under way must have retired before tensor memory is given up
        umma_commit(&bars->teardown);
        const long long t0 = clock64();
        while (!mbar_try_wait(&bars->teardown, 0)) {
          if (clock64() - t0 > kTimeoutCycles) break;
        }
      }
    }
    __syncwarp();
  } else {
    // ------------------------------------------------------------------ exponentials: a thread is a key against a share of the rows
    const int kt = warp / (4 * kShares), share = (warp >> 2) % kShares, key_in = kt * 128 + (warp & 3) * 32 + lane;
    const uint32_t d_addr = tmem_base + ((uint32_t)((warp & 3) * 32) << 16) + kt * 256 + share * kCols;
    auto all_draw = []() { asm volatile("bar.sync 1, %0;" ::"n"(kDrawWarps * 32) : "memory"); };
    bool ok = true;
    uint32_t count = 0;
    for (long long n = blockIdx.x; n < units; n += gridDim.x) {
      const WeighUnit u = unit_of(n);
      const int key = u.key0 + key_in, rows = u.seq.rows * in.group;
      float total = 0.0f;
      for (int t = u.tile0; t < u.tile1 && ok; ++t, ++count) {
        const uint32_t stage = count % kStages, slot = count & 1u;
        // the row's numbers come by way of the fetchers, the scores from the tensor core
        ok = mbar_wait_warp(&bars->q_full[stage], (count / kStages) & 1u, ctl) && mbar_wait_warp(&bars->d_full[kt][slot], (count >> 1) & 1u, ctl);
        if (!ok) break;
        tc_fence_after();
        const float* less = row_less + stage * 128 + share * kCols;
        const int* seen = row_seen + stage * 128 + share * kCols;
        // rows that are not there, or do not see all of the keys
        const bool edge = (t + 1) * kKvWeighRows > rows ||
                          kv_seen(u.seq.len, u.seq.rows, in.causal_block, t * kKvWeighRows / in.group) < u.key0 + (kt + 1) * 128;
        const float2 scale2 = make_float2(in.scale_log2, in.scale_log2);
        float2 sum = make_float2(0.0f, 0.0f);
#pragma unroll
        for (int c0 = 0; c0 < kCols; c0 += 32) {
          uint32_t x[32];
          tmem_ld32(d_addr + slot * 128 + c0, x);
          tmem_ld_wait();
          if (c0 + 32 == kCols) {  // all read
            tc_fence_before();
            __syncwarp();
            if (lane == 0) mbar_arrive(&bars->d_empty[kt][slot]);
          }
#pragma unroll
          for (int i = 0; i < 16; ++i) {
            const float2 l = *reinterpret_cast<const float2*>(less + c0 + 2 * i);
            float2 y = __ffma2_rn(make_float2(__uint_as_float(x[2 * i]), __uint_as_float(x[2 * i + 1])), scale2, l);
            y = make_float2(fast_exp2(y.x), fast_exp2(y.y));
            if (edge) {
              const int2 s = *reinterpret_cast<const int2*>(seen + c0 + 2 * i);
              y = make_float2(key < s.x ? y.x : 0.0f, key < s.y ? y.y : 0.0f);
            }
            sum = __fadd2_rn(sum, y);
          }
        }
        __syncwarp();
        if (lane == 0) mbar_arrive(&bars->q_empty[stage]);
        total += sum.x + sum.y;  // (a tile's own sum first: no number is added to more than a few dozen times its size in turn)
      }
      // the threads of a key, in their order
      if (share > 0) meet[(share - 1) * kBlock + key_in] = total;
      all_draw();
      bool mine = share == 0 && key < u.seq.len;
      if (share == 0) {
#pragma unroll
        for (int i = 1; i < kShares; ++i) total += meet[(i - 1) * kBlock + key_in];
      }
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
      all_draw();  // what was met with may be written again
    }
  }
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  if (warp == kIssuer) tmem_dealloc(tmem_base, 512);
}

template <int kHd, int kKind, int kTiles>
cudaError_t start_tiles(const litevggt_kv_cache& c, const litevggt_kv_batch& b, const KvWeighing& w, cudaStream_t s) {
  using Shape = WeighShape<kHd, kTiles>;
  static_assert(Shape::kSmemBytes <= 227 * 1024, "");
  auto kernel = kv_weigh_tiles_kernel<kHd, kKind, kTiles>;
  static std::atomic<unsigned long long> done{0};
  const cudaError_t e = set_max_dynamic_smem_once(reinterpret_cast<const void*>(kernel), Shape::kSmemBytes, done);
  if (e != cudaSuccess) return e;
  const WeighLists lists{reinterpret_cast<const long long*>(b.base + b.o_tiles_at), b.weigh.parts, reinterpret_cast<int*>(b.base + b.o_weigh_joins),
                         reinterpret_cast<float*>(b.base + b.o_weigh_sums)};
  const long long units = b.weigh.items * b.weigh.parts;
  return launch(kernel, dim3((unsigned)std::min(units, (long long)c.num_sms)), kWeighThreads, (size_t)Shape::kSmemBytes, s, c.pool, kv_arrays(b), w, lists,
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
  // A warp's run: as short as the chip allows, but no shorter than a unit.
  const long long warps = std::min(units, (long long)c.num_sms * 16), per_warp = (units + warps - 1) / warps;
  const unsigned blocks = (unsigned)(((units + per_warp - 1) / per_warp + kWeighWarps - 1) / kWeighWarps);
  const WeighLists lists{reinterpret_cast<const long long*>(b.base + b.o_few_at), 1, nullptr, nullptr};
  ++*launches;
  return by_kind(c, [&](auto hd, auto kind) {
    constexpr int kHd = decltype(hd)::value, kKind = decltype(kind)::value;
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
