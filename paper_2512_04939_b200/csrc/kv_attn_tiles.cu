// Attention of chunks over a paged K/V cache on the 5th-generation tensor cores.
//   o_i = sum_j p_ij v_j / sum_j p_ij,   p_ij = 2^(c q_i k_j - m_i)  for the keys j that row i sees
// A piece is up to 256 rows (two tiles of 128) of one sequence and K/V head against a range of keys in tiles of 128; heads
// that share K and V are rows side by side, so their keys come once.  One CTA per SM works off the pieces of its share.
//
// Tensor memory (512 columns): S of both tiles, 128 columns each; the rest is output.
//   head dim 64:  a tile's 128 keys are two streams of 64, each with four softmax warps of its own (one thread = one row), its
//                 own reference and its own 64 columns of output: the two halves of a row never speak to each other until
//                 the end of the piece, where they are weighed against one another.  16 softmax warps.
//   head dim 128: one stream of 128 keys a tile, 128 columns of output.  8 softmax warps; here the tensor cores are the bound.
// P (bf16 pairs) goes over the start of the stream's own columns of S and is the second product's A operand.  The instructions
// of a tile retire in order: Q K^T of the next key tile is issued behind the P V that reads the columns it writes, and when
// its scores are reported, that P V has retired as well.  So a softmax warp that finds a row's maximum far above its reference
// may scale the row's output right there.  While one tile waits for its products, the other's softmax runs.
//
// Warps: softmax; two MMA issuers (one per tile); one TMA producer; one that looks after V, or four that widen codes:
//   bf16  K comes by TMA straight into its swizzled tile, V too; a tile of V that holds keys which some rows do not see passes
//         the V warp: what no row sees becomes zero (a page's tail may hold anything, and 0 * NaN is NaN), and values that
//         are not finite are taken out; the softmax adds them to the rows that see them.
//   E4M3  codes and exponents come by bulk copies into a ring of their own; the four warps widen them to the same tiles, exactly.
#include "exp2.cuh"
#include "kv_cache.h"
#include "kv_quant.cuh"

namespace lv {

namespace {

constexpr int kTileKeys = 128;
#ifndef LV_KV_POLY
#define LV_KV_POLY 0
#endif

template <int kHd, bool kNarrow>
struct TiShape {
  static constexpr int kStreams = kHd == 64 ? 2 : 1;  // of a tile
  static constexpr int kKeys = kTileKeys / kStreams;  // of a stream's step
  static constexpr int kSoftmaxWarps = 8 * kStreams;
  static constexpr int kHelpers = kNarrow ? 4 : 1;
  static constexpr int kThreads = (kSoftmaxWarps + 3 + kHelpers) * 32;
  static constexpr int kStages = kHd == 64 ? (kNarrow ? 3 : 4) : 2;
  static constexpr int kRaw = kNarrow ? (kHd == 64 ? 3 : 1) : 0;
  static constexpr int kSubBytes = 128 * 128;             // 128 rows of 64 channels
  static constexpr int kTileBytes = kSubBytes * kHd / 64; // of Q, K or V
  static constexpr int kRawBytes = kTileKeys * kHd + kTileKeys;
  static constexpr uint32_t kColO = 256;
  static constexpr int kPolyPairs = LV_KV_POLY;  // of the 16 pairs of 32 scores, on the FMA pipes
  static constexpr int kSmemBytes = 2 * kTileBytes + 2 * kStages * kTileBytes + 2 * kRaw * kRawBytes + (kStreams == 2 ? 8192 : 0) + 512 + 1024;
};

template <int kStages, int kRaw>
struct TiBarriers {
  uint64_t k_full[kStages], k_empty[kStages], v_full[kStages], v_empty[kStages], v_land[kStages];
  uint64_t raw_full[2][kRaw > 0 ? kRaw : 1], raw_empty[2][kRaw > 0 ? kRaw : 1];  // [K, V]
  uint64_t q_ready[2], s_full[2][2], p_ready[2][2], o_done[2], teardown[2];
  uint32_t tmem_base, abort_flag;
  int taken_out[2];  // a piece (its number + 1, by its parity) whose V held values that are not finite where not all rows see them
  int last_of_join;
};

__device__ __forceinline__ void bulk_load(void* smem_dst, const void* src, uint32_t bytes, uint64_t* bar) {
  asm volatile("cp.async.bulk.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1], %2, [%3];" ::"r"(smem_u32(smem_dst)),
               "l"(src), "r"(bytes), "r"(smem_u32(bar))
               : "memory");
}
__device__ __forceinline__ void named_barrier(int id, int threads) { asm volatile("bar.sync %0, %1;" ::"r"(id), "r"(threads) : "memory"); }

// A row's reference moves to its maximum when a step's probabilities add up to more than kLate, and then if that maximum lies
// more than kSlack above it (base-2 units).  So no probability is over 2^20, which bf16 and sums in 32 bits hold as well
// as 1; what a maximum 2^20 above the reference takes from the other end is keys under 2^-106 of it.
constexpr float kLate = 1048576.0f, kSlack = 4.0f;

// Of `from`, the latest loads (up to one a slot) have landed; they must before the shared memory is given up.
template <int kSlots>
__device__ __forceinline__ void drain(uint64_t* full, uint32_t issued, uint32_t* status) {
  for (uint32_t i = 0; i < (issued < (uint32_t)kSlots ? issued : (uint32_t)kSlots); ++i) {
    const uint32_t at = issued - 1 - i;
    const long long t0 = clock64();
    while (!mbar_try_wait(&full[at % kSlots], (at / kSlots) & 1u)) {
      if (clock64() - t0 > kTimeoutCycles) { atomicOr(status, kStatusTimeout); break; }
    }
  }
}

struct Ring {
  int slot = 0;
  uint32_t phase = 0;
  template <int kSlots>
  __device__ __forceinline__ void next() {
    if (++slot == kSlots) { slot = 0; phase ^= 1u; }
  }
};

// A piece as every role sees it.
struct Job {
  KvPiece p;
  KvSeq q;
  int tile0, tiles;  // key tiles
  int min_seen;      // keys below it are seen by every row
  int max_seen;      // keys from it on by none
};
__device__ __forceinline__ Job job_of(const KvLaunch& work, const KvArrays& arrays, const KvAttend& at, int id) {
  Job j;
  j.p = work.pieces[id];
  j.q = arrays.seqs[j.p.seq];
  j.tile0 = j.p.key0 / kTileKeys;
  j.tiles = (j.p.key1 - j.p.key0 + kTileKeys - 1) / kTileKeys;
  j.min_seen = kv_seen(j.q.len, j.q.rows, at.causal_block, j.p.row0 / at.group);
  j.max_seen = kv_seen(j.q.len, j.q.rows, at.causal_block, (j.p.row0 + j.p.rows - 1) / at.group);
  return j;
}
// Key tiles of the piece that row tile t takes part in.
__device__ __forceinline__ int tiles_of(const Job& j, const KvAttend& at, int t) {
  if (j.p.rows <= t * 128) return 0;
  const int last = j.p.row0 + min(j.p.rows, (t + 1) * 128) - 1;
  const int seen = min(kv_seen(j.q.len, j.q.rows, at.causal_block, last / at.group), j.p.key1);
  return seen > j.p.key0 ? (seen - j.p.key0 + kTileKeys - 1) / kTileKeys : 0;
}

template <int kHd, bool kNarrow>
__global__ void __launch_bounds__(TiShape<kHd, kNarrow>::kThreads, 1)
kv_attn_tiles_kernel(const __grid_constant__ CUtensorMap k_map, const __grid_constant__ CUtensorMap v_map, KvPool pool, KvArrays arrays,
                     KvLaunch work, KvAttend at, uint32_t* status) {
  using Shape = TiShape<kHd, kNarrow>;
  constexpr int kStreams = Shape::kStreams, kStages = Shape::kStages, kRaw = Shape::kRaw, kRawSlots = kRaw > 0 ? kRaw : 1, kSubs = kHd / 64;
  constexpr int kTileBytes = Shape::kTileBytes, kSubBytes = Shape::kSubBytes;
  extern __shared__ uint8_t smem_raw[];
  uint8_t* smem_q = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~uintptr_t(1023));
  uint8_t* smem_k = smem_q + 2 * kTileBytes;
  uint8_t* smem_v = smem_k + kStages * kTileBytes;
  uint8_t* smem_codes = smem_v + kStages * kTileBytes;  // [K, V][slot] codes, then exponents
  float2* smem_ml = reinterpret_cast<float2*>(smem_codes + 2 * kRaw * Shape::kRawBytes);  // [parity][tile][stream][row]
  using Barriers = TiBarriers<kStages, kRaw>;
  Barriers* bars = reinterpret_cast<Barriers*>(smem_ml + (kStreams == 2 ? 1024 : 0));
  static_assert(sizeof(Barriers) <= 512, "");

  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  if (threadIdx.x == 0) {
    for (int i = 0; i < kStages; ++i) {
      mbar_init(&bars->k_full[i], kNarrow ? Shape::kHelpers : 1);
      mbar_init(&bars->k_empty[i], 2);
      mbar_init(&bars->v_full[i], Shape::kHelpers);
      mbar_init(&bars->v_empty[i], 2);
      mbar_init(&bars->v_land[i], 1);
    }
    for (int i = 0; i < (kRaw > 0 ? kRaw : 1); ++i)
      for (int x = 0; x < 2; ++x) {
        mbar_init(&bars->raw_full[x][i], 1);
        mbar_init(&bars->raw_empty[x][i], Shape::kHelpers);
      }
    for (int t = 0; t < 2; ++t) {
      mbar_init(&bars->q_ready[t], 4 * kStreams);
      mbar_init(&bars->s_full[t][0], 1);
      mbar_init(&bars->s_full[t][1], 1);
      mbar_init(&bars->p_ready[t][0], 4);
      mbar_init(&bars->p_ready[t][1], 4);
      mbar_init(&bars->o_done[t], 1);
      mbar_init(&bars->teardown[t], 1);
      bars->taken_out[t] = 0;
    }
    mbar_fence_init();
    bars->abort_flag = 0;
    if constexpr (!kNarrow) {
      tma_prefetch_desc(&k_map);
      tma_prefetch_desc(&v_map);
    }
  }
  constexpr int kIssuer = Shape::kSoftmaxWarps, kProducer = kIssuer + 2, kHelper = kIssuer + 3;
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
  const int id0 = work.first[blockIdx.x], id_end = work.first[blockIdx.x + 1];

  if (warp == kProducer) {
    // ------------------------------------------------------------------ TMA producer: lane i fetches a tile's i-th page
    Ring ring;
    uint32_t issued[2] = {0, 0};
    bool ok = true;
    const int per_tile = kTileKeys >> pool.page_shift;
    for (int id = id0; id < id_end && ok; ++id) {
      const Job job = job_of(work, arrays, at, id);
      for (int j = 0; j < job.tiles && ok; ++j) {
        const int key = (job.tile0 + j) * kTileKeys;
        const int n = min(per_tile, (job.q.len - key + pool.page_size - 1) >> pool.page_shift);
        long long row = 0;  // of the pool
        if (lane < n) {
          const long long page = arrays.pages[job.q.page0 + (key >> pool.page_shift) + lane];
          row = (page * pool.kv_heads + job.p.kv_head) * pool.page_size;
        }
#pragma unroll
        for (int x = 0; x < 2; ++x) {
          uint64_t *full, *empty;
          uint32_t bytes;
          if constexpr (kNarrow) {
            full = &bars->raw_full[x][ring.slot], empty = &bars->raw_empty[x][ring.slot];
            bytes = (uint32_t)(n * pool.page_size * (kHd + 1));
          } else {
            full = x == 0 ? &bars->k_full[ring.slot] : &bars->v_land[ring.slot];
            empty = x == 0 ? &bars->k_empty[ring.slot] : &bars->v_empty[ring.slot];
            bytes = (uint32_t)(n * pool.page_size * kHd * 2);
          }
          ok = ok && mbar_wait_warp(empty, ring.phase ^ 1u, ctl);
          if (!ok) break;
          if (lane == 0) mbar_expect_tx(full, bytes);
          __syncwarp();
          if (lane < n) {
            if constexpr (kNarrow) {
              uint8_t* dst = smem_codes + (x * kRaw + ring.slot) * Shape::kRawBytes;
              bulk_load(dst + lane * pool.page_size * kHd, (x == 0 ? pool.k : pool.v) + row * kHd, (uint32_t)(pool.page_size * kHd), full);
              bulk_load(dst + kTileKeys * kHd + lane * pool.page_size, (x == 0 ? pool.k_exp : pool.v_exp) + row, (uint32_t)pool.page_size, full);
            } else {
              uint8_t* dst = (x == 0 ? smem_k : smem_v) + ring.slot * kTileBytes + lane * pool.page_size * 128;
#pragma unroll
              for (int s = 0; s < kSubs; ++s) tma_load_2d(dst + s * kSubBytes, x == 0 ? &k_map : &v_map, full, s * 64, (int)row);
            }
          }
          __syncwarp();
          ++issued[x];
        }
        if constexpr (kNarrow) ring.next<kRawSlots>();
        else ring.next<kStages>();
      }
    }
    if (lane == 0) {  // every load has landed before the CTA may go
      drain<kNarrow ? kRawSlots : kStages>(kNarrow ? bars->raw_full[0] : bars->k_full, issued[0], status);
      drain<kNarrow ? kRawSlots : kStages>(kNarrow ? bars->raw_full[1] : bars->v_land, issued[1], status);
    }
    __syncwarp();
  } else if (warp == kIssuer || warp == kIssuer + 1) {
    // ------------------------------------------------------------------ MMA issuer of row tile t
    if (elect_one()) {
      const int t = warp - kIssuer;
      constexpr uint32_t idesc_qk = umma_idesc_bf16(128, Shape::kKeys, false, false);
      constexpr uint32_t idesc_pv = umma_idesc_bf16(128, kHd, false, true);
      const uint32_t s_col = tmem_base + t * 128;
      const uint32_t o_col = tmem_base + Shape::kColO + t * kStreams * kHd;
      const uint64_t q_desc = smem_desc_sw128(smem_u32(smem_q + t * kTileBytes), 16, 1024);
      const uint64_t k_desc0 = smem_desc_sw128(smem_u32(smem_k), 16, 1024);
      const uint64_t v_desc0 = smem_desc_sw128(smem_u32(smem_v), kSubBytes, 1024);  // 64 channels further on: the next sub-tile
      auto slot_at = [&](int slot) { return (uint64_t)((slot * kTileBytes) >> 4); };
      auto issue_qk = [&](int c, int slot) {
#pragma unroll
        for (int k = 0; k < kHd / 16; ++k) {
          const uint64_t in_tile = (uint64_t)(((k >> 2) * kSubBytes + (k & 3) * 32) >> 4);
          umma_ss(s_col + c * 64, q_desc + in_tile, k_desc0 + slot_at(slot) + (uint64_t)(c * 512) + in_tile, idesc_qk, k != 0 ? 1u : 0u);
        }
        umma_commit(&bars->s_full[t][c]);
      };
      Ring ring;
      uint32_t step = 0, round = 0;
      bool ok = true;
      for (int id = id0; id < id_end && ok; ++id) {
        const Job job = job_of(work, arrays, at, id);
        const int mine = tiles_of(job, at, t);
        if (mine > 0) {
          ok = mbar_wait(&bars->q_ready[t], round & 1u, ctl) && mbar_wait(&bars->k_full[ring.slot], ring.phase, ctl);
          if (!ok) break;
          tc_fence_after();
#pragma unroll
          for (int c = 0; c < kStreams; ++c) issue_qk(c, ring.slot);
          umma_commit(&bars->k_empty[ring.slot]);
        }
        for (int j = 0; j < job.tiles && ok; ++j) {
          Ring next = ring;
          next.next<kStages>();
          if (j < mine) {
            ok = mbar_wait(&bars->v_full[ring.slot], ring.phase, ctl);
            if (ok && j + 1 < mine) ok = mbar_wait(&bars->k_full[next.slot], next.phase, ctl);
#pragma unroll
            for (int c = 0; c < kStreams; ++c) {
              ok = ok && mbar_wait(&bars->p_ready[t][c], step & 1u, ctl);
              if (!ok) break;
              tc_fence_after();
#pragma unroll
              for (int k = 0; k < Shape::kKeys / 16; ++k)
                umma_ts(o_col + c * kHd, s_col + c * 64 + k * 8, v_desc0 + slot_at(ring.slot) + (uint64_t)(((c * 64 + k * 16) * 128) >> 4),
                        idesc_pv, (j | k) != 0 ? 1u : 0u);
              if (j + 1 < mine) issue_qk(c, next.slot);  // where these probabilities were
            }
            if (!ok) break;
            umma_commit(&bars->v_empty[ring.slot]);
            if (j + 1 < mine) umma_commit(&bars->k_empty[next.slot]);
            else umma_commit(&bars->o_done[t]);
            ++step;
          } else {  // tiles that the other rows see
            ok = mbar_wait(&bars->k_full[ring.slot], ring.phase, ctl) && mbar_wait(&bars->v_full[ring.slot], ring.phase, ctl);
            if (!ok) break;
            mbar_arrive(&bars->k_empty[ring.slot]);
            mbar_arrive(&bars->v_empty[ring.slot]);
          }
          ring = next;
        }
        round += mine > 0 ? 1u : 0u;
      }
      if (!ok) {  // what is under way must have retired before tensor memory is given up
        umma_commit(&bars->teardown[t]);
        const long long t0 = clock64();
        while (!mbar_try_wait(&bars->teardown[t], 0)) {
          if (clock64() - t0 > kTimeoutCycles) break;
        }
      }
    }
    __syncwarp();
  } else if (warp >= kHelper) {
    // ------------------------------------------------------------------ V (and what is held in codes)
    Ring ring, raw;
    bool ok = true;
    for (int id = id0; id < id_end && ok; ++id) {
      const Job job = job_of(work, arrays, at, id);
      for (int j = 0; j < job.tiles && ok; ++j) {
        const int key = (job.tile0 + j) * kTileKeys;
        const int end = job.max_seen - key;           // rows of the tile from here on are seen by nobody
        const int part = max(job.min_seen - key, 0);  // and from here on not by everybody
        if constexpr (kNarrow) {
          const int tid = threadIdx.x - kHelper * 32;
#pragma unroll 1
          for (int x = 0; x < 2; ++x) {
            ok = ok && mbar_wait_warp(&bars->raw_full[x][raw.slot], raw.phase, ctl);
            ok = ok && mbar_wait_warp(x == 0 ? &bars->k_empty[ring.slot] : &bars->v_empty[ring.slot], ring.phase ^ 1u, ctl);
            if (!ok) break;
            const uint8_t* codes = smem_codes + (x * kRaw + raw.slot) * Shape::kRawBytes;
            const uint8_t* exps = codes + kTileKeys * kHd;
            uint8_t* tile = (x == 0 ? smem_k : smem_v) + ring.slot * kTileBytes;
            bool bad = false;
            constexpr int kPerRow = kHd / 16;  // 16 codes at a time
#pragma unroll 4
            for (int i = 0; i < kPerRow; ++i) {
              const int piece = i * 128 + tid, r = piece / kPerRow, ch = piece % kPerRow;
              const uint4 w4 = *reinterpret_cast<const uint4*>(codes + piece * 16);
              const uint32_t byte = exps[r], w[4] = {w4.x, w4.y, w4.z, w4.w};
              const KvFactor f = kv_factor(byte);
              uint32_t v[8];
#pragma unroll
              for (int e = 0; e < 4; ++e) {
                v[2 * e] = mul_bf16x2(kv_code_bits(__byte_perm(w[e], 0u, 0x1404)), f.first * 0x10001u);
                v[2 * e + 1] = mul_bf16x2(kv_code_bits(__byte_perm(w[e], 0u, 0x3424)), f.first * 0x10001u);
              }
              if (kv_needs_second(byte)) {
#pragma unroll
                for (int e = 0; e < 8; ++e) v[e] = mul_bf16x2(v[e], f.second * 0x10001u);
                if (x == 1 && r >= part) {
#pragma unroll
                  for (int e = 0; e < 8; ++e) {
                    if ((v[e] & 0x7f80u) == 0x7f80u) v[e] &= 0xffff0000u, bad = bad || r < end;
                    if ((v[e] & 0x7f800000u) == 0x7f800000u) v[e] &= 0x0000ffffu, bad = bad || r < end;
                  }
                }
              }
              if (x == 1 && r >= end) {
#pragma unroll
                for (int e = 0; e < 8; ++e) v[e] = 0u;
              }
              uint8_t* row = tile + (ch >> 2) * kSubBytes + r * 128;
              *reinterpret_cast<uint4*>(row + (((2 * ch) & 7) ^ (r & 7)) * 16) = make_uint4(v[0], v[1], v[2], v[3]);
              *reinterpret_cast<uint4*>(row + (((2 * ch + 1) & 7) ^ (r & 7)) * 16) = make_uint4(v[4], v[5], v[6], v[7]);
            }
            if (bad) *reinterpret_cast<volatile int*>(&bars->taken_out[id & 1]) = id + 1;
            fence_proxy_async_shared();
            __syncwarp();
            if (lane == 0) {
              mbar_arrive(x == 0 ? &bars->k_full[ring.slot] : &bars->v_full[ring.slot]);
              mbar_arrive(&bars->raw_empty[x][raw.slot]);
            }
          }
          raw.next<kRawSlots>();
        } else {
          ok = mbar_wait_warp(&bars->v_land[ring.slot], ring.phase, ctl);
          if (!ok) break;
          if (part < kTileKeys) {
            bool bad = false;
            for (int i = part * 8 + lane; i < kTileKeys * 8; i += 32)
#pragma unroll
              for (int s = 0; s < kSubs; ++s) {
                uint4* at_row = reinterpret_cast<uint4*>(smem_v + ring.slot * kTileBytes + s * kSubBytes) + i;
                if (i >= end * 8) {
                  *at_row = make_uint4(0u, 0u, 0u, 0u);
                  continue;
                }
                const uint4 x = *at_row;
                uint32_t v[4] = {x.x, x.y, x.z, x.w};
                bool here = false;
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                  if ((v[e] & 0x7f80u) == 0x7f80u) v[e] &= 0xffff0000u, here = true;
                  if ((v[e] & 0x7f800000u) == 0x7f800000u) v[e] &= 0x0000ffffu, here = true;
                }
                if (here) *at_row = make_uint4(v[0], v[1], v[2], v[3]);
                bad = bad || here;
              }
            if (bad) *reinterpret_cast<volatile int*>(&bars->taken_out[id & 1]) = id + 1;
            fence_proxy_async_shared();
          }
          __syncwarp();
          if (lane == 0) mbar_arrive(&bars->v_full[ring.slot]);
        }
        ring.next<kStages>();
      }
    }
  } else {
    // ------------------------------------------------------------------ softmax: a thread is a row (of a stream)
    const int t = warp / (4 * kStreams), c = (warp >> 2) % kStreams, quarter = warp & 3;
    const int r = quarter * 32 + lane;  // within the tile
    const uint32_t lane_base = (uint32_t)(quarter * 32) << 16;
    const uint32_t s_addr = tmem_base + lane_base + t * 128 + c * 64;
    const uint32_t o_tile = tmem_base + lane_base + Shape::kColO + t * kStreams * kHd, o_addr = o_tile + c * kHd;
    uint32_t step = 0, round = 0;
    bool ok = true;
    for (int id = id0; id < id_end; ++id) {
      const Job job = job_of(work, arrays, at, id);
      const int mine = tiles_of(job, at, t);
      const bool live = t * 128 + r < job.p.rows;
      const int row = job.p.row0 + (live ? t * 128 + r : 0), token = row / at.group;
      const int seen = kv_seen(job.q.len, job.q.rows, at.causal_block, token);
      const long long out_row = (long long)(job.q.row0 + token) * at.q_heads + job.p.kv_head * at.group + row % at.group;
      if (mine > 0) {
        // the queries before have been read: o_done came behind their last product
        const __nv_bfloat16* src = at.q + (job.q.row0 + token) * at.q_stride.row + (job.p.kv_head * at.group + row % at.group) * at.q_stride.head;
        constexpr int kChunks = kHd / 8 / kStreams;  // 16 bytes each; streams share a row
        uint4 x[kChunks];
#pragma unroll
        for (int i = 0; i < kChunks; ++i) x[i] = live ? ldg16(src + (c * kChunks + i) * 8) : make_uint4(0u, 0u, 0u, 0u);
#pragma unroll
        for (int i = 0; i < kChunks; ++i) {
          const int ch = c * kChunks + i;
          *reinterpret_cast<uint4*>(smem_q + t * kTileBytes + (ch >> 3) * kSubBytes + r * 128 + ((ch & 7) ^ (r & 7)) * 16) = x[i];
        }
        fence_proxy_async_shared();
        __syncwarp();
        if (lane == 0) mbar_arrive(&bars->q_ready[t]);
      }
      float top = -INFINITY, ref = 0.0f;  // ref: top once that is finite
      float2 sum = make_float2(0.0f, 0.0f);
      const int first_seen = __shfl_sync(0xffffffffu, live ? seen : 0x7fffffff, 0);  // rows of a warp see ever more

      // One step: 64 or 128 scores of the row.  With kEdge some rows of the warp do not see all of its keys.
      constexpr int kGroups = Shape::kKeys / 32;
      bool unset = true;  // a row of the warp has no reference yet
      auto take_step = [&](auto edge_constant, int key, bool first) {
        constexpr bool kEdge = decltype(edge_constant)::value;
        auto load = [&](int g, uint32_t (&s)[32]) {
          tmem_ld32(s_addr + g * 32, s);
          tmem_ld_wait();
          if constexpr (kEdge) {
#pragma unroll
            for (int i = 0; i < 32; ++i)
              if (key + g * 32 + i >= seen) s[i] = 0xff800000u;
          }
        };
        // The row's maximum becomes its reference where it lies far above the present one.
        auto refer = [&]() {
          float most = -INFINITY;
#pragma unroll 1
          for (int g = 0; g < kGroups; ++g) {
            uint32_t s[32];
            load(g, s);
            float m[4];
#pragma unroll
            for (int i = 0; i < 4; ++i) {
              const uint32_t* x = &s[8 * i];
              m[i] = fmax3(__uint_as_float(x[0]), __uint_as_float(x[1]), __uint_as_float(x[2]));
              m[i] = fmax3(m[i], __uint_as_float(x[3]), __uint_as_float(x[4]));
              m[i] = fmax3(m[i], __uint_as_float(x[5]), __uint_as_float(x[6]));
            }
            most = fmax3(most, fmax3(m[0], m[1], __uint_as_float(s[7])), fmax3(m[2], m[3], __uint_as_float(s[15])));
            most = fmax3(most, __uint_as_float(s[23]), __uint_as_float(s[31]));
          }
          most *= at.scale_log2;
          const bool move = most > top + kSlack;
          const float factor = move ? (top == -INFINITY ? 0.0f : fast_exp2(ref - most)) : 1.0f;
          if (move) {
            top = ref = most;
            sum.x *= factor;
            sum.y *= factor;
          }
          unset = __any_sync(0xffffffffu, top == -INFINITY);
          if (!first) {
#pragma unroll 1
            for (int g = 0; g < kHd / 16; ++g) {
              uint32_t o[16];
              tmem_ld16(o_addr + g * 16, o);
              tmem_ld_wait();
#pragma unroll
              for (int i = 0; i < 16; ++i) o[i] = __float_as_uint(__uint_as_float(o[i]) * factor);
              tmem_st16(o_addr + g * 16, o);
            }
          }
        };
        // Only a row's first keys are asked for their maximum.  After that its probabilities are taken under the reference
        // that it has; they tell by themselves when it has fallen too far behind, before anything has been put in the place of
        // the scores: then the reference moves and they are taken again.
        uint32_t p[kGroups][16];
        float2 more;
#pragma unroll 1
        for (bool again = false;; again = true) {
          if (unset || again) refer();
          const float2 scale2 = make_float2(at.scale_log2, at.scale_log2), ref2 = make_float2(-ref, -ref);
          more = make_float2(0.0f, 0.0f);
#pragma unroll
          for (int g = 0; g < kGroups; ++g) {
            uint32_t s[32];
            load(g, s);
#pragma unroll
            for (int i = 0; i < 16; ++i) {
              float2 x = __ffma2_rn(make_float2(__uint_as_float(s[2 * i]), __uint_as_float(s[2 * i + 1])), scale2, ref2);
              if (i < Shape::kPolyPairs) {
                x = poly_exp2_pair(make_float2(fminf(fmax_nan(x.x, -126.0f), 120.0f), fminf(fmax_nan(x.y, -126.0f), 120.0f)));
              } else {
                x = make_float2(fast_exp2(x.x), fast_exp2(x.y));
              }
              p[g][i] = pack_bf16(x.x, x.y);
              // Where a row may see few keys, the sum is that of the rounded probabilities, so that their rounding changes only
              // what a key weighs among the others; elsewhere it averages out.
              more = __fadd2_rn(more, kEdge ? make_float2(bf16_lo(p[g][i]), bf16_hi(p[g][i])) : x);
            }
          }
          if (again || !__any_sync(0xffffffffu, !(more.x + more.y <= kLate))) break;
        }
        sum = __fadd2_rn(sum, more);
#pragma unroll
        for (int g = 0; g < kGroups; ++g) tmem_st16(s_addr + g * 16, p[g]);
      };
      for (int j = 0; j < mine && ok; ++j, ++step) {
        ok = mbar_wait_warp(&bars->s_full[t][c], step & 1u, ctl);
        if (!ok) break;
        tc_fence_after();
        const int key = (job.tile0 + j) * kTileKeys + c * 64;
        if (key + Shape::kKeys > first_seen) take_step(std::true_type{}, key, j == 0);
        else take_step(std::false_type{}, key, j == 0);
        tmem_st_wait();
        tc_fence_before();
        __syncwarp();
        if (lane == 0) mbar_arrive(&bars->p_ready[t][c]);
      }
      if (mine > 0) {
        ok = ok && mbar_wait_warp(&bars->o_done[t], round & 1u, ctl);
        ++round;
        tc_fence_after();
      }

      // ---------------------------------------------------------------- the piece's rows
      float row_sum = sum.x + sum.y, m = top, weight[kStreams];
      weight[0] = 1.0f;
      if constexpr (kStreams == 2) {
        float2* ml = smem_ml + ((id & 1) * 2 + t) * 256;
        ml[c * 128 + r] = make_float2(top, row_sum);
        named_barrier(1 + t * 4 + quarter, 64);
        const float2 a = ml[r], b = ml[128 + r];
        m = fmaxf(a.x, b.x);
        const float m_use = m == -INFINITY ? 0.0f : m;
        weight[0] = a.x == -INFINITY ? 1.0f : fast_exp2(a.x - m_use);  // without a key so far: its sum and rows are zero
        weight[1] = b.x == -INFINITY ? 1.0f : fast_exp2(b.x - m_use);
        row_sum = a.y * weight[0] + b.y * weight[1];
      }
      const bool bad = *reinterpret_cast<volatile int*>(&bars->taken_out[id & 1]) == id + 1;
      const bool whole = job.p.slot < 0;
      const float inverse = whole ? (seen > 0 ? 1.0f / row_sum : 0.0f) : 1.0f;
      constexpr int kMine = kHd / kStreams / 32;  // groups of 32 channels of this thread
#pragma unroll 1
      for (int g = 0; g < kMine; ++g) {
        const int ch0 = (kStreams == 2 ? c : g) * 32;
        float acc[32];
        if (mine > 0) {
          uint32_t o[32];
          tmem_ld32(o_tile + ch0, o);
          tmem_ld_wait();
#pragma unroll
          for (int i = 0; i < 32; ++i) acc[i] = __uint_as_float(o[i]) * weight[0];
          if constexpr (kStreams == 2) {
            tmem_ld32(o_tile + kHd + ch0, o);
            tmem_ld_wait();
#pragma unroll
            for (int i = 0; i < 32; ++i) acc[i] = fmaf(__uint_as_float(o[i]), weight[kStreams - 1], acc[i]);
          }
        } else {
#pragma unroll
          for (int i = 0; i < 32; ++i) acc[i] = 0.0f;
        }
        if (bad && live) {
          // values that were taken out of V, for the rows that see them
          for (int key = max(job.p.key0, job.min_seen); key < min(job.p.key1, seen); ++key) {
            const long long page = arrays.pages[job.q.page0 + (key >> pool.page_shift)];
            const long long at_row = (page * pool.kv_heads + job.p.kv_head) * pool.page_size + (key & (pool.page_size - 1));
            for (int i = 0; i < 32; ++i) {
              float v;
              if constexpr (kNarrow) {
                const uint32_t byte = pool.v_exp[at_row];
                const KvFactor f = kv_factor(byte);
                uint32_t w = mul_bf16x2(kv_code_bits((uint32_t)pool.v[at_row * kHd + ch0 + i] << 8), f.first);
                if (kv_needs_second(byte)) w = mul_bf16x2(w, f.second);
                v = bf16_lo(w);
              } else {
                v = __bfloat162float(reinterpret_cast<const __nv_bfloat16*>(pool.v)[at_row * kHd + ch0 + i]);
              }
              if (!(fabsf(v) < INFINITY)) {
#pragma unroll
                for (int e = 0; e < 32; ++e)
                  if (e == i) acc[e] += v;
              }
            }
          }
        }
        if (whole) {
          if (live) {
            uint4* dst = reinterpret_cast<uint4*>(at.out + out_row * kHd + ch0);
#pragma unroll
            for (int i = 0; i < 4; ++i) {
              float v[8];
#pragma unroll
              for (int e = 0; e < 8; ++e) v[e] = seen > 0 ? acc[8 * i + e] * inverse : 0.0f;
              dst[i] = make_uint4(pack_bf16(v[0], v[1]), pack_bf16(v[2], v[3]), pack_bf16(v[4], v[5]), pack_bf16(v[6], v[7]));
            }
          }
        } else {
          // rows side by side, four channels of each at a time: a warp's store is 512 bytes in a row
          float4* dst = reinterpret_cast<float4*>(work.rows) + ((size_t)job.p.slot * (kHd / 4) + ch0 / 4) * 256 + t * 128 + r;
#pragma unroll
          for (int i = 0; i < 8; ++i) __stcg(dst + i * 256, make_float4(acc[4 * i], acc[4 * i + 1], acc[4 * i + 2], acc[4 * i + 3]));
        }
      }
      tc_fence_before();
      if (!whole) {
        if (c == 0) __stcg(reinterpret_cast<float2*>(work.sums) + (size_t)job.p.slot * 256 + t * 128 + r, make_float2(m, row_sum));
        // whoever comes last adds the parts up, in their order
        __threadfence();
        named_barrier(9, Shape::kSoftmaxWarps * 32);
        if (threadIdx.x == 0) {
          const int before = atomicAdd(work.joins + job.p.join, 1);
          bars->last_of_join = before == job.p.parts - 1;
          if (before == job.p.parts - 1) work.joins[job.p.join] = 0;
        }
        named_barrier(9, Shape::kSoftmaxWarps * 32);
        if (*reinterpret_cast<volatile int*>(&bars->last_of_join) != 0 && live) {
          __threadfence();
          const float2* ml = reinterpret_cast<const float2*>(work.sums) + (size_t)job.p.first_slot * 256 + t * 128 + r;
          float joint = -INFINITY, l = 0.0f;
          for (int w = 0; w < job.p.parts; ++w) joint = fmaxf(joint, __ldcg(ml + (size_t)w * 256).x);
          const float use = joint == -INFINITY ? 0.0f : joint;
          auto weight_of = [&](float x) { return x == -INFINITY ? 1.0f : fast_exp2(x - use); };
          for (int w = 0; w < job.p.parts; ++w) {
            const float2 x = __ldcg(ml + (size_t)w * 256);
            l += x.y * weight_of(x.x);
          }
          const float inv = 1.0f / l;
#pragma unroll 1
          for (int g = 0; g < kMine; ++g) {
            const int ch0 = (kStreams == 2 ? c : g) * 32;
            float acc[32];
#pragma unroll
            for (int i = 0; i < 32; ++i) acc[i] = 0.0f;
            for (int w = 0; w < job.p.parts; ++w) {
              const float wt = weight_of(__ldcg(ml + (size_t)w * 256).x);
              const float4* part = reinterpret_cast<const float4*>(work.rows) + ((size_t)(job.p.first_slot + w) * (kHd / 4) + ch0 / 4) * 256 + t * 128 + r;
#pragma unroll
              for (int i = 0; i < 8; ++i) {
                const float4 x = __ldcg(part + i * 256);
                acc[4 * i] = fmaf(x.x, wt, acc[4 * i]);
                acc[4 * i + 1] = fmaf(x.y, wt, acc[4 * i + 1]);
                acc[4 * i + 2] = fmaf(x.z, wt, acc[4 * i + 2]);
                acc[4 * i + 3] = fmaf(x.w, wt, acc[4 * i + 3]);
              }
            }
            uint4* dst = reinterpret_cast<uint4*>(at.out + out_row * kHd + ch0);
#pragma unroll
            for (int i = 0; i < 4; ++i) {
              float v[8];
#pragma unroll
              for (int e = 0; e < 8; ++e) v[e] = seen > 0 ? acc[8 * i + e] * inv : 0.0f;
              dst[i] = make_uint4(pack_bf16(v[0], v[1]), pack_bf16(v[2], v[3]), pack_bf16(v[4], v[5]), pack_bf16(v[6], v[7]));
            }
          }
        }
        named_barrier(9, Shape::kSoftmaxWarps * 32);  // last_of_join has been read
      }
    }
  }
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  if (warp == kIssuer) tmem_dealloc(tmem_base, 512);
}

template <int kHd, bool kNarrow>
cudaError_t start(const litevggt_kv_cache& c, const litevggt_kv_batch& b, const KvAttend& a, cudaStream_t s) {
  using Shape = TiShape<kHd, kNarrow>;
  auto kernel = kv_attn_tiles_kernel<kHd, kNarrow>;
  static std::atomic<unsigned long long> done{0};
  const cudaError_t e = set_max_dynamic_smem_once(reinterpret_cast<const void*>(kernel), Shape::kSmemBytes, done);
  if (e != cudaSuccess) return e;
  const KvLaunch work = kv_launch(b, b.tiles, b.at_tiles);
  return launch(kernel, dim3((unsigned)work.workers), Shape::kThreads, (size_t)Shape::kSmemBytes, s, c.k_map, c.v_map, c.pool, kv_arrays(b),
                work, a, c.status);
}

}  // namespace

cudaError_t launch_kv_attn_tiles(const litevggt_kv_cache& c, const litevggt_kv_batch& b, const KvAttend& a, cudaStream_t s, int* launches) {
  const bool narrow = c.cfg.dtype == LITEVGGT_KV_E4M3;
  ++*launches;
  if (c.cfg.head_dim == 64) return narrow ? start<64, true>(c, b, a, s) : start<64, false>(c, b, a, s);
  return narrow ? start<128, true>(c, b, a, s) : start<128, false>(c, b, a, s);
}

}  // namespace lv
