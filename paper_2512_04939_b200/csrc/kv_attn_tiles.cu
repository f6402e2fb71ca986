// Attention of chunks over a paged K/V cache on the 5th-generation tensor cores.
//   o_i = sum_j p_ij v_j / sum_j p_ij,   p_ij = 2^(c q_i k_j - m_i)  for the keys j that row i sees
// A piece is up to 256 rows (two tiles of 128) of one sequence and K/V head against a range of keys in tiles of 128; heads
// that share K and V are rows side by side, so their keys come once.  One CTA per SM works off the pieces of its share.
//
// Two threads share a row, 64 of a key tile's 128 keys each (streams; 16 softmax warps).  At head dim 64 the special-function unit
// is the bound (16 exponentials a clock against 256 tensor operations for each), so all else is kept away from it and from
// the issue slots: Q is an operand from tensor memory, and the second product's B operand carries a column of ones, so that
// the tensor core adds up the bf16 probabilities that it multiplies.  At head dim 128 the tensor cores are the bound, and their
// memory is full with S and O: Q comes from shared memory, the threads add up their own probabilities.
// A row's reference is its maximum in the piece's first key tile, and it stays: p may grow to 2^60 in bf16 and 32-bit sums as
// well as stay below 1.  Where it grows more (the row's sum tells, at the end of the piece), or where the first key tile leaves a row
// without a reference, the piece is done again when all others are through, with one sweep for the maxima first; then a row's largest
// score is taken off before the scale, so scores may be as large as 32 bits hold.
// Tensor memory (512 columns): S of both tiles, 128 columns each; O of both, 80 columns (64 channels, the sum, 15 unused) or 128;
// at head dim 64 Q of both, 32 columns.  P (bf16 pairs) goes over the start of the stream's own columns of S and is the second
// product's A operand.  The instructions of a tile retire in order: a stream's next Q K^T is issued behind the P V that reads the
// columns it writes.
//
// Warps: softmax; two MMA issuers (one per tile), a TMA producer, one that looks after V; for codes eight that widen them:
//   bf16  K and V come by TMA straight into their swizzled tiles; in V what no row sees becomes zero (a page's tail may
//         hold anything, and 0 * NaN is NaN).  Values that are not finite, of keys that some rows see and others do not, make
//         the piece come again, and then they are taken out here and added to the rows that see them.
//   E4M3  codes and exponents come by bulk copies into a ring of their own; the eight warps widen them to the same tiles,
//         exactly, and look after V on the way.
//
// 2048 rows over 83,280 keys, 699 GFLOP: head dim 64 (16 heads) 786 us, 889 TFLOP/s; head dim 128 (8 heads) 630 us, 1110; over E4M3
// 946 us and 780.  In bursts; under the 1 kW cap, which all of them reach, head dim 64 makes 750.  What bounds them (2048 rows over 10,410
// keys): head dim 64 the special-function unit, 67 % of it with set-up and all, beside 44 % of the issue slots and 43 % of the
// tensor cores; head dim 128 nothing alone (tensor cores and special-function unit 52 %): a stream waits for its own products, and Q's
// share of shared memory's bandwidth is taken twice a key tile; codes the issue slots (60 % and 58 %), at 72 registers a thread, of which
// 334 and 506 bytes are spilled (bf16 76 and 176, at 96).  A piece of 17 rows, which a frame of 1,041 leaves behind four of 256, runs
// like one of 128: most of its softmax warps take exponentials of rows that do not exist.
// Tried and left: one product of 128 columns for both streams' scores at head dim 128 (643 -> 649 us, 98 -> 109 at 10,410 keys: the
// streams then wait for each other); the first 32 keys' probabilities handed over ahead of the others (no change); registers
// moved between warps by setmaxnreg (no function may be called then, and the waits in line cost more than the registers
// gave); rows by way of shared memory and the end of a piece as a function (3 % each: registers of the sweep); V looked
// through by the producer, without a warp of its own (1 % at head dim 64, 5 % over codes).
#include "exp2.cuh"
#include "kv_cache.h"
#include "kv_handoff.h"
#include "kv_quant.cuh"

namespace lv {

namespace {

constexpr int kTileKeys = 128;
constexpr int kStreams = 2;                  // of a tile: a row's two threads
constexpr int kSoftmaxWarps = 8 * kStreams;
constexpr int kKeys = kTileKeys / kStreams;  // of a stream's step

template <int kHd, bool kNarrow>
struct TiShape {
  static constexpr bool kOnes = kHd == 64;    // the tensor core adds up the rows, and Q is in its memory
  // Of the 16 pairs of 32 scores, this many take their exponentials on the FMA pipes: 16 issue slots and more for 16 clocks of the
  // special-function unit.  That pays where this unit is the bound, and not beside codes that are widened.  2048 rows over 83,280
  // keys, none / 1 / 2 / 4 pairs: head dim 64 802 / 786 / 787 / 797 us, E4M3 946 / 952 / 966 / 1006; head dim 128 629 / 636 / 643 /
  // 640, E4M3 780 / 785 / 801 / 819.
  static constexpr int kPolyPairs = kOnes && !kNarrow ? 2 : 0;
  static constexpr int kHelpers = kNarrow ? 8 : 1;
  static constexpr int kThreads = (kSoftmaxWarps + 4 + (kNarrow ? 8 : 0)) * 32;
  static constexpr int kStages = kHd == 64 ? (kNarrow ? 3 : 4) : 2;
  static constexpr int kRaw = kNarrow ? (kHd == 64 ? 3 : 1) : 0;
  static constexpr int kSubBytes = 128 * 128;             // 128 rows of 64 channels
  static constexpr int kTileBytes = kSubBytes * kHd / 64; // of Q, K or V
  static constexpr int kRawBytes = kTileKeys * kHd + kTileKeys;
  static constexpr int kOnesBytes = kOnes ? 16 * 128 : 0;
  static constexpr uint32_t kColO = 256, kOCols = kOnes ? 80 : 128, kColQ = 416;
  static constexpr int kQBytes = kOnes ? 0 : 2 * kTileBytes;
  static constexpr int kSmemBytes = kQBytes + 2 * kStages * kTileBytes + kOnesBytes + 2 * kRaw * kRawBytes + 512 + 1024;
};

template <int kStages, int kRaw>
struct TiBarriers {
  uint64_t k_full[kStages], k_empty[kStages], v_full[kStages], v_empty[kStages], v_land[kStages];
  uint64_t raw_full[2][kRaw > 0 ? kRaw : 1], raw_empty[2][kRaw > 0 ? kRaw : 1];  // [K, V]
  uint64_t q_ready[2], s_full[2][2], p_ready[2][2], o_done[2], teardown[2];
  uint32_t tmem_base, abort_flag;
  int any_again, last_of_join;
};
// Marks of a piece, in device memory: the row tiles and the warps that look after V may be several short pieces apart.
constexpr int kAgain = 1;     // it has to be done again
constexpr int kTakenOut = 2;  // its V held values that are not finite where not all rows see them
__device__ __forceinline__ void set_mark(int* mark, int value) { *reinterpret_cast<volatile int*>(mark) = value; }
__device__ __forceinline__ int get_mark(const int* mark) { return *reinterpret_cast<const volatile int*>(mark); }

// 2^x for a pair of arguments on the FMA pipes: the nearest whole number n goes into the exponent field, a cubic gives the
// power of the rest (relative error 7.5e-5, far below the rounding to bf16).  The arguments are held to [-125, 125] first, where
// rounding to n leaves a rest of at most a half: what lies below comes out as next to nothing, what lies above as a number that no row's
// sum overlooks.  So does a NaN, which passes these bounds: the integer sum makes the largest finite number of it.
__device__ __forceinline__ float hold(float x) {
  float y;
  asm("{\n\t.reg .f32 t;\n\tmin.NaN.f32 t, %1, 0f42FA0000;\n\tmax.NaN.f32 %0, t, 0fC2FA0000;\n\t}" : "=f"(y) : "f"(x));
  return y;
}
__device__ __forceinline__ float2 poly_exp2_held(float2 x) { return poly_exp2_pair(make_float2(hold(x.x), hold(x.y))); }
// What a row's sum has to stay below.
constexpr float kSumLimit = 1.152921504606847e18f;  // 2^60

__device__ __forceinline__ void bulk_load(void* smem_dst, const void* src, uint32_t bytes, uint64_t* bar) {
  asm volatile("cp.async.bulk.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1], %2, [%3];" ::"r"(smem_u32(smem_dst)),
               "l"(src), "r"(bytes), "r"(smem_u32(bar))
               : "memory");
}
__device__ __forceinline__ void named_barrier(int id, int threads) { asm volatile("bar.sync %0, %1;" ::"r"(id), "r"(threads) : "memory"); }

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
__device__ __forceinline__ Job job_of(const KvLaunch& work, const KvAttend& at, int id) {
  Job j;
  j.p = work.pieces[id];
  j.q = j.p.seq;
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
  constexpr bool kOnes = Shape::kOnes;
  constexpr int kStages = Shape::kStages, kRaw = Shape::kRaw, kRawSlots = kRaw > 0 ? kRaw : 1, kSubs = kHd / 64;
  constexpr int kTileBytes = Shape::kTileBytes, kSubBytes = Shape::kSubBytes;
  extern __shared__ uint8_t smem_raw[];
  uint8_t* smem_q = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~uintptr_t(1023));
  uint8_t* smem_k = smem_q + Shape::kQBytes;
  uint8_t* smem_v = smem_k + kStages * kTileBytes;
  uint8_t* smem_ones = smem_v + kStages * kTileBytes;
  uint8_t* smem_codes = smem_ones + Shape::kOnesBytes;  // [K, V][slot] codes, then exponents
  using Barriers = TiBarriers<kStages, kRaw>;
  Barriers* bars = reinterpret_cast<Barriers*>(smem_codes + 2 * kRaw * Shape::kRawBytes);
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
    }
    mbar_fence_init();
    bars->abort_flag = 0;
    bars->any_again = 0;
    if constexpr (!kNarrow) {
      tma_prefetch_desc(&k_map);
      tma_prefetch_desc(&v_map);
    }
  }
  // The block behind V whose first column is 1 and whose other columns are 0: 16 key rows laid out like a V tile, the last 16
  // of the second product's 80 columns.  Every instruction's descriptor carries the stride from its own V rows to it.
  if (kOnes && threadIdx.x < Shape::kOnesBytes / 16) {
    const int r = threadIdx.x >> 3, chunk = threadIdx.x & 7;
    reinterpret_cast<uint4*>(smem_ones)[threadIdx.x] = make_uint4(chunk == (r & 7) ? 0x00003f80u : 0u, 0u, 0u, 0u);
    fence_proxy_async_shared();
  }
  constexpr int kIssuer = kSoftmaxWarps, kProducer = kIssuer + 2, kHelper = kNarrow ? kIssuer + 4 : kIssuer + 3;
  if (warp == kIssuer) {
    tmem_alloc(&bars->tmem_base, 512);
    tmem_relinquish();
  }
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tmem_base = bars->tmem_base;
  const WaitCtl ctl{&bars->abort_flag, status};
  if (threadIdx.x == 0) asm volatile("prefetch.global.L1 [%0];" ::"l"(work.pieces + blockIdx.x));
  wait_for_previous_kernel();

  enum Mode { kFast = 0, kMaxima = 1, kCareful = 2 };
  // Steps of a row tile in which some rows do not see all keys, and all of a piece that is done again: those that reach past
  // edge_from.  Rows may see few keys there, so their probabilities go in as two bf16 numbers each, in two products; elsewhere
  // what one of them rounds averages out.
  auto edge_from = [&](const Job& job, int mode, int t) {
    return mode == kCareful ? 0 : kv_seen(job.q.len, job.q.rows, at.causal_block, (job.p.row0 + t * 128) / at.group);
  };
  // Every role goes over the CTA's pieces; and a second time over those whose reference did not do, twice each: once for the
  // maxima, once for the rows.
  auto pieces = [&](auto run) {
    for (int id = (int)blockIdx.x; id >= 0;) {
      id = run(id, kFast);
      __syncwarp();
    }
    named_barrier(10, Shape::kThreads);
    if (*reinterpret_cast<volatile int*>(&bars->any_again) == 0) return;
    for (int id = (int)blockIdx.x; id >= 0; id = work.pieces[id].next)
      if (get_mark(work.again + id) != 0) {
        run(id, kMaxima);
        __syncwarp();
        run(id, kCareful);
        __syncwarp();
      }
  };

  if (warp == kProducer) {
    // ------------------------------------------------------------------ TMA producer: lane i fetches a tile's i-th page
    Ring ring;
    uint32_t issued[2] = {0, 0};
    bool ok = true;
    const int per_tile = kTileKeys >> pool.page_shift;
    pieces([&](int id, int) -> int {
      const Job job = job_of(work, at, id);
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
      return job.p.next;
    });
    if (lane == 0) {  // every load has landed before the CTA may go
      drain<kNarrow ? kRawSlots : kStages>(kNarrow ? bars->raw_full[0] : bars->k_full, issued[0], status);
      drain<kNarrow ? kRawSlots : kStages>(kNarrow ? bars->raw_full[1] : bars->v_land, issued[1], status);
    }
    __syncwarp();
  } else if (warp == kIssuer || warp == kIssuer + 1) {
    // ------------------------------------------------------------------ MMA issuer of row tile t: one lane
    const int t = warp - kIssuer;
    constexpr uint32_t idesc_qk = umma_idesc_bf16(128, kKeys, false, false);
    constexpr uint32_t idesc_pv = umma_idesc_bf16(128, Shape::kOCols, false, true);
    const uint32_t s_col = tmem_base + t * 128, o_col = tmem_base + Shape::kColO + t * Shape::kOCols, q_col = tmem_base + Shape::kColQ + t * 32;
    const uint64_t q_desc = smem_desc_sw128(smem_u32(smem_q + t * kTileBytes), 16, 1024);
    const uint64_t k_desc0 = smem_desc_sw128(smem_u32(smem_k), 16, 1024);
    // V's next 64 columns: the ones, behind the ring, or the next sub-tile.  x 16-byte units into the ring the stride to the
    // ones (bits 16-29) shrinks by what the address grows.
    const uint64_t v_desc0 = smem_desc_sw128(smem_u32(smem_v), kOnes ? kStages * kTileBytes : kSubBytes, 1024);
    auto v_desc_at = [&](uint32_t x) { return kOnes ? v_desc0 + x - ((uint64_t)x << 16) : v_desc0 + x; };
    auto issue_qk = [&](int c, int slot) {
#pragma unroll
      for (int k = 0; k < kHd / 16; ++k) {
        const uint64_t in_tile = (uint64_t)(((k >> 2) * kSubBytes + (k & 3) * 32) >> 4);
        const uint64_t k_desc = k_desc0 + (uint64_t)((slot * kTileBytes) >> 4) + (uint64_t)(c * 512) + in_tile;
        if constexpr (kOnes) umma_ts(s_col + c * 64, q_col + k * 8, k_desc, idesc_qk, k != 0 ? 1u : 0u);
        else umma_ss(s_col + c * 64, q_desc + in_tile, k_desc, idesc_qk, k != 0 ? 1u : 0u);
      }
      umma_commit(&bars->s_full[t][c]);
    };
    Ring ring;
    uint32_t step = 0, round = 0;
    bool ok = true;
    pieces([&](int id, int mode) -> int {
      if (elect_one()) {  // the same lane every time
        const Job job = job_of(work, at, id);
        const int mine = tiles_of(job, at, t), all_see = edge_from(job, mode, t);
        if (ok && mine > 0) {
          ok = mbar_wait(&bars->q_ready[t], round & 1u, ctl) && mbar_wait(&bars->k_full[ring.slot], ring.phase, ctl);
          if (ok) {
            tc_fence_after();
#pragma unroll
            for (int c = 0; c < kStreams; ++c) issue_qk(c, ring.slot);
            umma_commit(&bars->k_empty[ring.slot]);
            // what the first product awaits beside its own stream, here, where it is not in the loop's way
            static_assert(kStreams == 2 && kv_awaits(0, 0, 1) && !kv_awaits(0, 1, 0) && !kv_awaits(1, 0, 1) && !kv_awaits(1, 1, 0), "");
            ok = mbar_wait(&bars->p_ready[t][1], step & 1u, ctl);
          }
        }
        for (int j = 0; j < job.tiles && ok; ++j) {
          Ring next = ring;
          next.next<kStages>();
          if (j < mine) {
            ok = mbar_wait(&bars->v_full[ring.slot], ring.phase, ctl);
#pragma unroll
            for (int c = 0; c < kStreams; ++c) {
              ok = ok && mbar_wait(&bars->p_ready[t][c], step & 1u, ctl);
              if (!ok) break;
              tc_fence_after();
              if (mode != kMaxima) {
#pragma unroll
                for (int k = 0; k < kKeys / 16; ++k)
                  umma_ts(o_col, s_col + c * 64 + k * 8, v_desc_at((uint32_t)((ring.slot * kTileBytes + (c * 64 + k * 16) * 128) >> 4)),
                          idesc_pv, (j | c | k) != 0 ? 1u : 0u);
                if ((job.tile0 + j) * kTileKeys + c * 64 + kKeys > all_see) {  // what the rounding left over
#pragma unroll
                  for (int k = 0; k < kKeys / 16; ++k)
                    umma_ts(o_col, s_col + c * 64 + 32 + k * 8, v_desc_at((uint32_t)((ring.slot * kTileBytes + (c * 64 + k * 16) * 128) >> 4)),
                            idesc_pv, 1u);
                }
              }
              if (j + 1 < mine) {
                if (c == 0 && !(ok = mbar_wait(&bars->k_full[next.slot], next.phase, ctl))) break;
                tc_fence_after();
                issue_qk(c, next.slot);  // where these probabilities were
              }
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
      return work.pieces[id].next;
    });
    __syncwarp();
    if (elect_one() && !ok) {  // what is under way must have retired before tensor memory is given up
      umma_commit(&bars->teardown[t]);
      const long long t0 = clock64();
      while (!mbar_try_wait(&bars->teardown[t], 0)) {
        if (clock64() - t0 > kTimeoutCycles) break;
      }
    }
    __syncwarp();
  } else if (warp >= kHelper) {
    // ------------------------------------------------------------------ V (and what is held in codes)
    Ring ring, raw;
    bool ok = true;
    pieces([&](int id, int mode) -> int {
      const Job job = job_of(work, at, id);
      for (int j = 0; j < job.tiles && ok; ++j) {
        const int key = (job.tile0 + j) * kTileKeys;
        const int end = job.max_seen - key;           // rows of the tile from here on are seen by nobody
        // and from here on not by everybody; that matters only where values are not finite, and then the piece comes again
        const int part = mode == kCareful ? max(job.min_seen - key, 0) : end;
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
#pragma unroll 2
            for (int i = 0; i < kPerRow / 2; ++i) {
              const int piece = i * 256 + tid, r = piece / kPerRow, ch = piece % kPerRow;
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
                if (x == 1 && r >= part && mode == kCareful) {
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
            if (bad) set_mark(work.again + id, kAgain | kTakenOut);
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
          if (min(part, end) < kTileKeys) {
            bool bad = false;
            for (int i = max(min(part, end), 0) * 8 + lane; i < kTileKeys * 8; i += 32)
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
            if (bad) set_mark(work.again + id, kAgain | kTakenOut);
            fence_proxy_async_shared();
          }
          __syncwarp();
          if (lane == 0) mbar_arrive(&bars->v_full[ring.slot]);
        }
        ring.next<kStages>();
      }
      return job.p.next;
    });
  } else if (warp >= kIssuer) {
    pieces([&](int id, int) { return work.pieces[id].next; });  // (beside the warps that widen codes there is nothing left for the fourth)
  } else {
    // ------------------------------------------------------------------ softmax: a thread is a row, or the half of one
    const int t = warp / (4 * kStreams), c = (warp >> 2) % kStreams, quarter = warp & 3;
    const int r = quarter * 32 + lane;  // within the tile
    const uint32_t lane_base = (uint32_t)(quarter * 32) << 16;
    const uint32_t s_addr = tmem_base + lane_base + t * 128 + c * 64;
    const uint32_t o_addr = tmem_base + lane_base + Shape::kColO + t * Shape::kOCols;
    uint32_t step = 0, round = 0;
    bool ok = true;
    float kept = -INFINITY;  // the row's largest score, from one sweep to the next
    // The queries, this thread's half row.  Those before have been read where o_done has come: it follows their last product.
    constexpr int kChunks = kHd / 16;  // of 16 bytes
    int given = -1;                    // the piece whose queries are there already
    auto read_q = [&](const Job& job, uint4 (&x)[kChunks]) {
      const bool live = t * 128 + r < job.p.rows;
      const int row = job.p.row0 + (live ? t * 128 + r : 0);
      const __nv_bfloat16* src = at.q + (job.q.row0 + row / at.group) * at.q_stride.row +
                                 (job.p.kv_head * at.group + row % at.group) * at.q_stride.head + c * (kHd / 2);
#pragma unroll
      for (int i = 0; i < kChunks; ++i) x[i] = live ? ldg16(src + i * 8) : make_uint4(0u, 0u, 0u, 0u);
    };
    auto give_q = [&](const uint4 (&x)[kChunks]) {
      if constexpr (kOnes) {
        uint32_t w[16];
#pragma unroll
        for (int i = 0; i < 4; ++i) w[4 * i] = x[i].x, w[4 * i + 1] = x[i].y, w[4 * i + 2] = x[i].z, w[4 * i + 3] = x[i].w;
        tmem_st16(tmem_base + lane_base + Shape::kColQ + t * 32 + c * 16, w);
        tmem_st_wait();
        tc_fence_before();
      } else {
#pragma unroll
        for (int i = 0; i < kChunks; ++i)
          *reinterpret_cast<uint4*>(smem_q + t * kTileBytes + c * kSubBytes + r * 128 + (i ^ (r & 7)) * 16) = x[i];
        fence_proxy_async_shared();
      }
      __syncwarp();
      if (lane == 0) mbar_arrive(&bars->q_ready[t]);
    };
    auto largest = [](const uint32_t (&s)[32]) {
      float m[4];
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const uint32_t* x = &s[8 * i];
        m[i] = fmax3(__uint_as_float(x[0]), __uint_as_float(x[1]), __uint_as_float(x[2]));
        m[i] = fmax3(m[i], __uint_as_float(x[3]), __uint_as_float(x[4]));
        m[i] = fmax3(m[i], __uint_as_float(x[5]), __uint_as_float(x[6]));
        m[i] = fmaxf(m[i], __uint_as_float(x[7]));
      }
      return fmaxf(fmax3(m[0], m[1], m[2]), m[3]);
    };
    pieces([&](int id, int mode) -> int {
      // What the sweep needs of the piece; the rest is read again behind it, where it does not hold registers.
      int mine, key_base, seen, all_see;
      bool live;
      {
        const Job job = job_of(work, at, id);
        mine = tiles_of(job, at, t);
        key_base = job.tile0 * kTileKeys + c * 64;
        live = t * 128 + r < job.p.rows;
        seen = kv_seen(job.q.len, job.q.rows, at.causal_block, (job.p.row0 + (live ? t * 128 + r : 0)) / at.group);
        all_see = edge_from(job, mode, t);
        if (mine > 0 && given != id) {
          uint4 x[kChunks];
          read_q(job, x);
          give_q(x);
        }
        given = -1;
      }
      float top = -INFINITY, ref = 0.0f;  // the row's reference; ref: what is subtracted of scaled scores, top where that is finite
      float2 sum = make_float2(0.0f, 0.0f);

      auto key_of = [&](int j) { return key_base + j * kTileKeys; };
      auto scores_in = [&]() {
        const bool in = mbar_wait_warp(&bars->s_full[t][c], step & 1u, ctl);
        if (in) tc_fence_after();
        return in;
      };
      auto give_p = [&]() {
        tmem_st_wait();
        tc_fence_before();
        __syncwarp();
        if (lane == 0) mbar_arrive(&bars->p_ready[t][c]);
      };
      // This thread's 64 scores of a step.  With kEdge some rows may not see all of its keys.
      uint32_t s[2][32];
      auto load = [&](bool edge, int key) {
        tmem_ld32(s_addr, s[0]);
        tmem_ld32(s_addr + 32, s[1]);
        tmem_ld_wait();
        if (edge) {
#pragma unroll
          for (int g = 0; g < 2; ++g)
#pragma unroll
            for (int i = 0; i < 32; ++i)
              if (key + g * 32 + i >= seen) s[g][i] = 0xff800000u;
        }
      };
      auto take_half = [&](auto edge_constant, int key) {
        constexpr bool kEdge = decltype(edge_constant)::value;
        load(kEdge, key);
        // Done again: less the largest score before anything is rounded, so that the largest probability is 1 whatever the scores' size.
        // (Scaled first, a maximum of 2^30 is rounded by up to 32, and 2^32 would be no probability.)
        const float less = kEdge && mode == kCareful && kept != -INFINITY ? -kept : 0.0f;
        const float2 scale2 = make_float2(at.scale_log2, at.scale_log2), ref2 = make_float2(-ref, -ref);
#pragma unroll
        for (int g = 0; g < 2; ++g) {
          uint32_t p[16], rest[kEdge ? 16 : 1];
#pragma unroll
          for (int i = 0; i < 16; ++i) {
            float2 x = make_float2(__uint_as_float(s[g][2 * i]), __uint_as_float(s[g][2 * i + 1]));
            if constexpr (kEdge) x = __fadd2_rn(x, make_float2(less, less));
            x = __ffma2_rn(x, scale2, ref2);
            if (!kEdge && i < Shape::kPolyPairs) x = poly_exp2_held(x);
            else x = make_float2(fast_exp2(x.x), fast_exp2(x.y));
            if constexpr (kEdge) {
              // The upper half as it is, and the rest; never a rest of zero or less beside a probability, which an infinite value
              // would make a NaN of.
              p[i] = __byte_perm(__float_as_uint(x.x), __float_as_uint(x.y), 0x7632);
              rest[i] = pack_bf16(fmaf(x.x, 9.3e-10f, x.x - bf16_lo(p[i])), fmaf(x.y, 9.3e-10f, x.y - bf16_hi(p[i])));
            } else {
              p[i] = pack_bf16(x.x, x.y);
            }
            // the sum of what is multiplied: the rounded ones, or both parts
            if constexpr (!kOnes) sum = __fadd2_rn(sum, kEdge ? x : make_float2(bf16_lo(p[i]), bf16_hi(p[i])));
          }
          if constexpr (kEdge) tmem_st16(s_addr + 32 + g * 16, rest);
          tmem_st16(s_addr + g * 16, p);
        }
      };
      float most = -INFINITY;
      auto add_maximum = [&](int key) {
        load(key + kKeys > all_see, key);
        most = fmaxf(most, fmaxf(largest(s[0]), largest(s[1])));
      };
      // The two threads of a row tell each other a number, by way of two columns of tensor memory that nothing else writes before
      // both have read them.  Both come here whatever became of their waits.
      auto exchange = [&](uint32_t column, uint32_t apart, float own) {
        tmem_st1(column + c * apart, __float_as_uint(own));
        tmem_st_wait();
        tc_fence_before();
        named_barrier(1 + t * 4 + quarter, 64);
        tc_fence_after();
        uint32_t both[2];
        tmem_ld1(column, both[0]);
        tmem_ld1(column + apart, both[1]);
        tmem_ld_wait();
        return make_float2(__uint_as_float(both[0]), __uint_as_float(both[1]));  // in the same order for both
      };
      // They agree on its maximum: each where its part of the output before has been read; the next begins when both have handed over
      // probabilities (kv_awaits), and so have read what the other one left there.
      auto agree = [&]() {
        const float2 both = exchange(o_addr, kHd / 2, most);
        return fmaxf(both.x, both.y);
      };
      if (mine > 0) {
        if (mode == kFast) {
          ok = ok && scores_in();
          if (ok) add_maximum(key_of(0));
          top = agree() * at.scale_log2;
        } else if (mode == kMaxima) {
          for (int j = 0; j < mine && ok; ++j, ++step) {
            ok = scores_in();
            if (!ok) break;
            add_maximum(key_of(j));
            give_p();
          }
          kept = agree();
        } else {
          top = kept * at.scale_log2;
        }
        ref = top == -INFINITY || mode == kCareful ? 0.0f : top;
        if (mode != kMaxima) {
          for (int j = 0; j < mine && ok; ++j, ++step) {
            ok = scores_in();
            if (!ok) break;
            if (key_of(j) + kKeys > all_see) take_half(std::true_type{}, key_of(j));
            else take_half(std::false_type{}, key_of(j));
            give_p();
          }
        }
      }
      asm volatile("" ::: "memory");
      const Job job = job_of(work, at, id);
      const int row = job.p.row0 + (live ? t * 128 + r : 0), token = row / at.group;
      const long long out_row = (long long)(job.q.row0 + token) * at.q_heads + job.p.kv_head * at.group + row % at.group;
      float row_sum = sum.x + sum.y;
      if (mine > 0) {
        // The next piece's queries are under way while the last products are, and its first scores while the rows leave.  (At
        // head dim 64 that costs registers which the sweep has not got: 2.5 % at 2048 rows over 83,280 keys.)
        Job next = job;
        bool some = false;
        uint4 x[kChunks];
        if (!kOnes && mode == kFast && job.p.next >= 0) {
          next = job_of(work, at, job.p.next);
          some = tiles_of(next, at, t) > 0;
          if (some) read_q(next, x);
        }
        ok = ok && mbar_wait_warp(&bars->o_done[t], round & 1u, ctl);
        ++round;
        tc_fence_after();
        if (!kOnes && mode != kMaxima) {
          const float2 both = exchange(s_addr - c * 64, 64, row_sum);  // where the last scores were
          row_sum = both.x + both.y;
        }
        if (some) {
          give_q(x);
          given = job.p.next;
        }
      }
      if (mode == kMaxima) return 0;

      // ---------------------------------------------------------------- the piece's rows
      const bool has = live && seen > job.p.key0;  // the row sees keys of this piece
      if (kOnes && mine > 0) {
        uint32_t l;
        tmem_ld1(o_addr + 64, l);
        tmem_ld_wait();
        row_sum = has ? __uint_as_float(l) : 0.0f;
      }
      const bool whole = job.p.slot < 0;
      const float inverse = whole && seen > 0 ? 1.0f / row_sum : 1.0f;
      constexpr int kMine = kHd / kStreams / 32;  // groups of 32 channels of this thread
#pragma unroll 1
      for (int g = 0; g < kMine; ++g) {
        const int ch0 = (c * kMine + g) * 32;
        float acc[32];
        if (mine > 0) {
          uint32_t o[32];
          tmem_ld32(o_addr + ch0, o);
          tmem_ld_wait();
#pragma unroll
          for (int i = 0; i < 32; ++i) acc[i] = __uint_as_float(o[i]);
        } else {
#pragma unroll
          for (int i = 0; i < 32; ++i) acc[i] = 0.0f;
        }
        if (mode == kFast && has) {
          float zero = 0.0f;  // NaN where something is not finite
#pragma unroll
          for (int i = 0; i < 32; ++i) zero = fmaf(acc[i], 0.0f, zero);
          // (a row whose first key tile left it without a reference has none that other parts could be weighed against)
          if (!(top > -INFINITY && row_sum > 0.0f && row_sum < kSumLimit && zero == 0.0f)) {
            set_mark(work.again + id, kAgain);
            set_mark(&bars->any_again, 1);
          }
        }
        if (mode == kCareful && live && (get_mark(work.again + id) & kTakenOut) != 0) {
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
        if (c == 0) __stcg(reinterpret_cast<float2*>(work.sums) + (size_t)job.p.slot * 256 + t * 128 + r, make_float2(top, row_sum));
        // whoever comes last adds the parts up, in their order; a piece that is to be done again has not come
        __threadfence();
        named_barrier(9, kSoftmaxWarps * 32);
        if (threadIdx.x == 0) {
          int last = 0;
          if (mode == kCareful || *reinterpret_cast<volatile int*>(&bars->any_again) == 0 || get_mark(work.again + id) == 0) {
            last = atomicAdd(work.joins + job.p.join, 1) == job.p.parts - 1 ? 1 : 0;
            if (last) work.joins[job.p.join] = 0;
          }
          *reinterpret_cast<volatile int*>(&bars->last_of_join) = last;
        }
        named_barrier(9, kSoftmaxWarps * 32);
        if (*reinterpret_cast<volatile int*>(&bars->last_of_join) != 0 && live) {
          __threadfence();
          const float2* ml = reinterpret_cast<const float2*>(work.sums) + (size_t)job.p.first_slot * 256 + t * 128 + r;
          float joint = -INFINITY, l = 0.0f;
#pragma unroll 4
          for (int w = 0; w < job.p.parts; ++w) joint = fmaxf(joint, __ldcg(ml + (size_t)w * 256).x);
          const float use = joint == -INFINITY ? 0.0f : joint;
          auto weight_of = [&](float x) { return x == -INFINITY ? 1.0f : fast_exp2(x - use); };
#pragma unroll 4
          for (int w = 0; w < job.p.parts; ++w) {
            const float2 x = __ldcg(ml + (size_t)w * 256);
            l += x.y * weight_of(x.x);
          }
          const float inv = 1.0f / l;
#pragma unroll 1
          for (int g = 0; g < kMine; ++g) {
            const int ch0 = (c * kMine + g) * 32;
            float acc[32];
#pragma unroll
            for (int i = 0; i < 32; ++i) acc[i] = 0.0f;
#pragma unroll 2
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
        named_barrier(9, kSoftmaxWarps * 32);  // last_of_join has been read
      }
      return job.p.next;
    });
  }
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  if (warp == kIssuer) tmem_dealloc(tmem_base, 512);
  if (bars->any_again != 0) {
    if (threadIdx.x == 0)
      for (int id = (int)blockIdx.x; id >= 0; id = work.pieces[id].next) work.again[id] = 0;
  }
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
