// Attention of few rows over a paged K/V cache: single tokens, drafts of a few, heads that share K and V.
//   o_i = sum_j p_ij v_j / sum_j p_ij,   p_ij = 2^(c q_i k_j - m_i)  for the keys j that row i sees
// A piece is up to 16 rows of one sequence and K/V head (tokens times the query heads that share it) against a range of
// keys.  All that counts is that K and V come from memory once and at its full rate: 4 operations a byte at one row.
//
// Every warp has a ring of its own in shared memory, which it fills itself (TMA boxes of 16 keys, or bulk copies of codes) and
// which runs on from piece to piece, so that loads are under way whatever the warp is doing; the warps of a CTA take
// turns on a piece's keys, each with a softmax reference of its own, and meet once at its end.  From the ring the keys go
// straight into the fragments of mma.m16n8k16.  Which lane reads which bytes follows from the fragments:
//   S = Q K^T   B holds K[key = lane / 4][channels of lane % 4]: the four lanes of a key read 16 bytes each of its row, and the
//               contraction runs over the channels in the order in which they come (Q is loaded in the same order)
//   O = P V     B holds V[keys 2q, 2q + 1, 2q + 8, 2q + 9 with q = lane % 4][channel of lane / 4]: a lane reads 8 (or 16)
//               channels of those four keys and pairs them up with byte permutations; its accumulators' keys in S are the same
//               ones, so P goes from accumulator to operand without leaving the lane
// Codes are widened to f16, which takes one conversion for two of them.  Their powers of two stay outside: a key's scales its
// scores, a value's its probability; that product is the value's weight, relative to the row's largest.  Q goes to f16 under a
// power of two of its row (exact but for elements under 2^-30 of the row's largest, which keep steps of 2^-37 of it or less); weights
// have 11 bits there, not 8, down to 2^-21 of the row's largest or less, and fixed steps of 2^-31 of it or less below: where one key's value
// has a code of zero in a channel, keys of 2^-32 of its weight count as nothing there.
// Codes of 4 bits have a power of two for 32 channels.  Scores are sums of a block each in f16, brought together in 32 bits under the
// blocks' powers.  Values have to meet their powers before the product, which takes them in bf16, where codes and powers are exact: two
// keys' codes of a channel become a pair of the operand by permutations and one multiplication, without a conversion.
//
// One token of 16 heads of 64 over 260,250 keys in bf16: 176 us, 6.1 TB/s, the rate of a copy; 48 tokens of 16 heads of 128 over 1,100
// to 4,164 keys 166 us, 6.2 TB/s.  Codes of head dim 64 are bound by the work of widening them (a conversion takes as long as four of the
// other instructions; the ALU is 60 % busy): over 520,500 keys 201 us, 5.4 TB/s.  At head dim 128 nothing is over 30 % busy: two warps a
// scheduler, each with one chain of waits, conversions, products and exponentials (16 tokens, 8 query heads a K/V head, 35 us).
// Codes of 4 bits are half the bytes and about the same work, and it is the work that bounds them, issue slots and ALU: one token over
// 520,500 keys 197 us, 2.9 TB/s (335 with a conversion for every pair; values and weights in f16, under a power of two of the warp's,
// 4 % less, but then keys of 2^-32 of the heaviest one's weight count as nothing where its code is zero).
// (Straight from global memory into the fragments, without rings: 189, 307 and 404 us for the first three figures.  The scores by products of 8-bit operands, Q in two of them, which need no
// conversion of K in the source: 202 -> 220 us, sixteen tokens that share heads by eight 32.9 -> 33.2.)  Few keys: 4.8 us for 262, of which the latency of three dependent loads and the
// meeting of the parts are most.
#include "exp2.cuh"
#include "kv_cache.h"
#include "kv_mma.cuh"
#include "kv_quant.cuh"

namespace lv {

namespace {

__device__ __forceinline__ uint4 lds16(uint32_t addr) {
  uint4 v;
  asm volatile("ld.shared.v4.u32 {%0, %1, %2, %3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "r"(addr));
  return v;
}
__device__ __forceinline__ uint2 lds8(uint32_t addr) {
  uint2 v;
  asm volatile("ld.shared.v2.u32 {%0, %1}, [%2];" : "=r"(v.x), "=r"(v.y) : "r"(addr));
  return v;
}
// The powers of two of two neighbouring rows; infinity for one that is not finite.
__device__ __forceinline__ void power_pair(uint32_t addr, float (&p)[2]) {
  uint32_t v;
  asm volatile("{\n\t.reg .u16 h;\n\tld.shared.u16 h, [%1];\n\tcvt.u32.u16 %0, h;\n\t}" : "=r"(v) : "r"(addr));
  p[0] = __uint_as_float(v << 23 & 0x7f800000u);
  p[1] = __uint_as_float(v << 15 & 0x7f800000u);
}
__device__ __forceinline__ void bulk_load(uint32_t smem_dst, const void* src, uint32_t bytes, uint64_t* bar) {
  asm volatile("cp.async.bulk.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1], %2, [%3];" ::"r"(smem_dst), "l"(src),
               "r"(bytes), "r"(smem_u32(bar))
               : "memory");
}

// A row's reference is set this far above its maximum so far (base-2 units), and anew where a score exceeds it: probabilities are
// 2^-7 to 1 for the largest, never more, so that sums of values at the end of the range hold where they would for a reference that
// is the maximum.
constexpr float kFewAbove = 7.0f;
// Codes: a probability times its value's power of two is a weight, at most 2^120, and the product's operand is the
// weight times a power of two 2^k of its row.  That brings the largest weight to [2^7, 2^8) when it is set, and is set anew where
// one comes to more than 2^15 (f16 ends at 2^16).
constexpr int kFewWeight = 7, kFewMostShift = 118;
constexpr float kFewMostWeight = 32768.0f;
// E2M1, up to eight rows: where pieces have this many keys on average warps take 64 at a time (one token over 520,500 keys 210 -> 197 us, 48 sequences
// of 8192 with heads of 128 channels 352 -> 320); shorter pieces do not go evenly into warps' turns of 64 (48 tokens of 16 heads of 64 over up to 4164: 67 us with 32,
// 69 with 64; four drafts of two over 5000: 15.6, 17.4).
constexpr int kFewLongPiece = 4096;
__device__ __forceinline__ float power_of_two(int k) { return __int_as_float((k + 127) << 23); }
__device__ __forceinline__ int exponent_of(float x) { return (__float_as_int(x) >> 23) - 127; }

__device__ __forceinline__ uint32_t lds4(uint32_t addr) {
  uint32_t v;
  asm volatile("ld.shared.u32 %0, [%1];" : "=r"(v) : "r"(addr));
  return v;
}

// kLong: stages of 64 keys.
template <int kHd, int kKind, bool kHalf, bool kLong = false>
struct FewShape {
  static constexpr bool kNarrow = kKind == LITEVGGT_KV_E4M3, kFour = kKind == LITEVGGT_KV_E2M1;
  static constexpr bool kMoves = kHalf && !kFour;             // whether the accumulators' empty halves are left out of the registers
  static constexpr int kParts = kMoves ? 2 : 4;               // registers of a lane and tile of accumulators
  static constexpr int kBlocks = kFour ? kHd / 32 : 1;        // of channels that have a power of two of their own
  using Row = KvRow<kHd, kKind>;
  // Rings of 9 to 25 KB a warp.  Codes of head dim 64 take so much work for a byte that sixteen warps an SM serve them
  // better than eight with more registers (one token over 520,500: 216 us against 241 to 283); those of head dim 128 spill
  // under 128 registers (sixteen tokens that share heads by eight: 36 us against 49).  Stages of 32 keys in 4 bits: at head dim 128 what
  // a stage costs beside its keys is as much again (48 sequences of 8192 keys: 442 us with 16, 367 with 32).
  static constexpr int kCtas = kKind != LITEVGGT_KV_BF16 && kHd == 64 ? 2 : 1;  // per SM
  static constexpr int kSubs = kLong ? 4 : kNarrow || kFour ? 2 : 128 / kHd;  // of 16 keys, of a stage
  static constexpr int kStages = kFour ? (kLong ? 2 : 4) : kNarrow || (kHd == 128 && !kHalf) ? 2 : 3;
  static constexpr int kRows = kHalf ? 8 : 16;
  static constexpr int kOutTiles = kHd / 8;
  static constexpr int kSubBytes = 16 * Row::kBytes;  // of K or V
  static constexpr int kExpBytes = (2 * kSubs * 16 * Row::kExps + 127) / 128 * 128;  // exponents [K, V][sub] of 16 rows
  static constexpr int kStageBytes = 2 * kSubs * kSubBytes + kExpBytes;              // [K, V][sub], exponents
  static constexpr int kRingBytes = kKvFewWarps * kStages * kStageBytes;
  static constexpr int kMergeBytes = kKvFewWarps * kRows * (kHd + 2) * 4;
  static constexpr int kSmemBytes = kRingBytes + kMergeBytes + 1024 + 320;
  static_assert(kKvFewWarps * kStages * 8 + 8 <= 320, "");
};

// kHalf: at most eight rows, so the lower half of every row tile is empty and takes no registers.
template <int kHd, int kKind, bool kHalf, bool kLong>
__global__ void __launch_bounds__(kKvFewWarps * 32, FewShape<kHd, kKind, kHalf, kLong>::kCtas)
kv_attn_few_kernel(const __grid_constant__ CUtensorMap k_map, const __grid_constant__ CUtensorMap v_map, KvPool pool, KvArrays arrays,
                   KvLaunch work, KvAttend at, uint32_t* status) {
  using Shape = FewShape<kHd, kKind, kHalf, kLong>;
  constexpr bool kNarrow = Shape::kNarrow, kFour = Shape::kFour;
  constexpr int kBlocks = Shape::kBlocks, kParts4 = Shape::kParts;
  constexpr int kRowBytes = Shape::Row::kBytes, kExps = Shape::Row::kExps;
  constexpr int kSubs = Shape::kSubs, kStages = Shape::kStages, kStageKeys = 16 * kSubs, kRound = kKvFewWarps * kStageKeys;
  constexpr int kHalves = kHalf ? 1 : 2;
  extern __shared__ uint8_t smem_raw[];
  uint8_t* smem = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~uintptr_t(1023));
  float* smem_o = reinterpret_cast<float*>(smem + Shape::kRingBytes);  // [warp][row][channel]
  float* smem_ml = smem_o + kKvFewWarps * Shape::kRows * kHd;          // [warp][row]{reference, sum}
  uint64_t* bars = reinterpret_cast<uint64_t*>(smem + Shape::kRingBytes + Shape::kMergeBytes);  // [warp][stage]
  uint32_t* flags = reinterpret_cast<uint32_t*>(bars + kKvFewWarps * kStages);                  // abort, last of a join
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int g = lane >> 2, q4 = lane & 3;
  if (threadIdx.x < kKvFewWarps * kStages) {
    mbar_init(&bars[threadIdx.x], 1);
    mbar_fence_init();
  }
  if (threadIdx.x == 0) flags[0] = 0;
  __syncthreads();
  const WaitCtl ctl{flags, status};
  uint64_t* full = bars + warp * kStages;
  const uint32_t ring = smem_u32(smem) + warp * kStages * Shape::kStageBytes;

  // ------------------------------------------------------------------ loads
  // The stage that is fetched next, and its piece; a lane's copy is one of K or V of 16 keys and 64 channels, or of the codes or
  // exponents of as many keys of the stage as lie in a page (every copy takes a dozen instructions, and codes are bound by them).  Its
  // page is looked up a stage ahead.
  constexpr int kParts = kExps > 0 ? 2 : kHd / 64, kCopies = kSubs * 2 * kParts, kStageShift = kSubs == 4 ? 6 : kSubs == 2 ? 5 : 4;
  static_assert(kExps == 0 || 1 << kStageShift == kStageKeys, "");
  const int run_shift = kExps > 0 ? min(kStageShift, pool.page_shift) : 4;  // of a copy's keys
  const int my_part = lane % kParts, my_x = (lane / kParts) & 1, my_sub = lane / (2 * kParts);
  int f_id = (int)blockIdx.x, f_key = 0, f_end = 0, f_head = 0, f_page0 = 0, f_page = 0, f_next = -1;
  uint32_t fetched = 0;
  auto look_up = [&]() {
    const int key = f_key + (my_sub << run_shift);
    if (lane < kCopies && key < f_end) f_page = arrays.pages[f_page0 + (key >> pool.page_shift)];
  };
  auto enter = [&]() {  // the first piece from f_id on that has keys for this warp
    while (f_id >= 0) {
      const KvPiece p = work.pieces[f_id];
      f_key = p.key0 + warp * kStageKeys;
      f_end = p.key1;
      f_next = p.next;
      if (f_key < f_end) {
        f_head = p.kv_head;
        f_page0 = p.seq.page0;
        look_up();
        return;
      }
      f_id = f_next;
    }
  };
  auto fetch = [&]() {
    if (f_id < 0) return;
    const uint32_t stage = fetched % kStages;
    uint64_t* bar = &full[stage];
    const int runs = min(kStageKeys >> run_shift, (f_end - f_key + (1 << run_shift) - 1) >> run_shift);
    if (lane == 0) mbar_expect_tx(bar, (uint32_t)(runs * (2 * (kRowBytes + kExps)) << run_shift));
    __syncwarp();
    if (lane < kCopies && my_sub < runs) {
      const int key = f_key + (my_sub << run_shift);
      const long long row = ((long long)f_page * pool.kv_heads + f_head) * pool.page_size + (key & (pool.page_size - 1));
      const uint32_t base = ring + stage * Shape::kStageBytes;
      if constexpr (kExps > 0) {
        const int at = my_x * kStageKeys + (my_sub << run_shift);  // row of the stage
        if (my_part == 0) bulk_load(base + at * kRowBytes, (my_x == 0 ? pool.k : pool.v) + row * kRowBytes, kRowBytes << run_shift, bar);
        else bulk_load(base + 2 * kSubs * Shape::kSubBytes + at * kExps, (my_x == 0 ? pool.k_exp : pool.v_exp) + row * kExps, kExps << run_shift, bar);
      } else {
        const uint32_t dst = base + (my_x * kSubs + my_sub) * Shape::kSubBytes + my_part * 2048;
        asm volatile("cp.async.bulk.tensor.2d.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1, {%3, %4}], [%2];" ::"r"(dst),
                     "l"(reinterpret_cast<uint64_t>(my_x == 0 ? &k_map : &v_map)), "r"(smem_u32(bar)), "r"(my_part * 64), "r"((int)row)
                     : "memory");
      }
    }
    ++fetched;
    f_key += kRound;
    if (f_key < f_end) {
      look_up();
    } else {
      f_id = f_next;
      enter();
    }
  };
  enter();  // (a batch's arrays were there before whatever kernel is still running)
  wait_for_previous_kernel();
  for (int i = 0; i < kStages; ++i) fetch();

  uint32_t taken = 0;
  bool ok = true;
  KvPiece piece;
  for (int id = (int)blockIdx.x; id >= 0; id = piece.next) {
    piece = work.pieces[id];
    const KvSeq seq = piece.seq;

    // ---------------------------------------------------------------- rows
    uint32_t qa[kHd / 16][2 * kHalves];
    float row_scale[kHalves];  // of the scores, in base-2 units
#pragma unroll
    for (int half = 0; half < kHalves; ++half) {
      // 16 bytes of a K row hold the channels of two contraction steps of 16 (bf16) or of four (codes of 8 bits); of 4 bits a lane reads
      // 4 bytes of every block, two steps, so that a step lies in one block
      constexpr int kRun = kNarrow ? 16 : 8;  // channels of a lane that lie side by side
      const int r = g + 8 * half;
      const bool live = r < piece.rows;
      const int at_row = piece.row0 + (live ? r : 0);
      const __nv_bfloat16* src =
          at.q + (seq.row0 + at_row / at.group) * at.q_stride.row + (piece.kv_head * at.group + at_row % at.group) * at.q_stride.head;
      uint32_t top = 0;
#pragma unroll
      for (int i = 0; i < kHd / (4 * kRun); ++i)
#pragma unroll
        for (int j = 0; j < kRun / 4; ++j) {
          uint2 w = make_uint2(0u, 0u);
          if (live) w = *reinterpret_cast<const uint2*>(src + (i * 4 + q4) * kRun + 4 * j);
          qa[i * (kRun / 4) + j][half] = w.x;
          qa[i * (kRun / 4) + j][kHalves + half] = w.y;
          top = __vmaxu2(top, __vmaxu2(w.x & 0x7fff7fffu, w.y & 0x7fff7fffu));
        }
      row_scale[half] = at.scale_log2;
      if constexpr (kNarrow || kFour) {
        top = max(top & 0xffffu, top >> 16);
        top = max(top, __shfl_xor_sync(0xffffffffu, top, 1));
        top = max(top, __shfl_xor_sync(0xffffffffu, top, 2));
        const float2 factors = f16_factor(top);
        const float factor = factors.x;
        row_scale[half] *= factors.y;
#pragma unroll
        for (int i = 0; i < kHd / 16; ++i)
#pragma unroll
          for (int j = 0; j < 2; ++j) {
            const uint32_t w = qa[i][j * kHalves + half];
            qa[i][j * kHalves + half] = pack_f16(bf16_lo(w) * factor, bf16_hi(w) * factor);
          }
      }
    }
    auto seen_by = [&](int r) { return kv_seen(seq.len, seq.rows, at.causal_block, (piece.row0 + r) / at.group); };
    const int all_see = min(seen_by(0), piece.key1);  // keys before this one are seen by every row
    const int seen[2] = {min(seen_by(g), piece.key1), min(seen_by(g + 8), piece.key1)};

    float o[Shape::kOutTiles][kParts4];
#pragma unroll
    for (int i = 0; i < Shape::kOutTiles; ++i)
#pragma unroll
      for (int j = 0; j < kParts4; ++j) o[i][j] = 0.0f;
    float limit[2] = {-INFINITY, -INFINITY}, ref[2] = {0.0f, 0.0f}, sum[2] = {0.0f, 0.0f};  // limit: ref, or that there is none yet
    // Codes: the rows' factors of the weights, which the output has in it.  (A power of infinity stands for a value that is not
    // finite, whose codes are zero: 0 * infinity = NaN.)
    [[maybe_unused]] float to[2] = {power_of_two(kFewMostShift), power_of_two(kFewMostShift)};

    // ---------------------------------------------------------------- sweep
    // One stage; with `edge` some rows do not see all of its keys, or not all of its keys are there.
    auto take = [&](auto edge_constant, int key, uint32_t base) {
      constexpr bool edge = decltype(edge_constant)::value;
      [[maybe_unused]] const uint32_t exps = base + 2 * kSubs * Shape::kSubBytes;
      // scores
      float sc[kSubs][2][4];
#pragma unroll
      for (int s = 0; s < kSubs; ++s)
#pragma unroll
        for (int t = 0; t < 2; ++t) {
          float c_block[kBlocks][4];  // sums of the blocks, or the one sum
#pragma unroll
          for (int b = 0; b < kBlocks; ++b) c_block[b][0] = c_block[b][1] = c_block[b][2] = c_block[b][3] = 0.0f;
          const int row = g + 8 * t;
          const uint32_t at_sub = base + s * Shape::kSubBytes;
          auto step = [&](int n, uint32_t b0, uint32_t b1) {
            float (&c)[4] = c_block[kFour ? n / 2 : 0];
            if constexpr (kHalf) mma_16816<kNarrow || kFour>(c, qa[n][0], 0u, qa[n][1], 0u, b0, b1);
            else mma_16816<kNarrow || kFour>(c, qa[n][0], qa[n][1], qa[n][2], qa[n][3], b0, b1);
          };
          if constexpr (kNarrow) {
#pragma unroll
            for (int i = 0; i < kHd / 64; ++i) {
              const uint4 x = lds16(at_sub + row * kHd + i * 64 + q4 * 16);
              const uint32_t w[4] = {x.x, x.y, x.z, x.w};
#pragma unroll
              for (int j = 0; j < 4; ++j) step(4 * i + j, widen_low(w[j]), widen_high(w[j]));
            }
          } else if constexpr (kFour) {
#pragma unroll
            for (int i = 0; i < kBlocks; ++i) {
              uint32_t x[4];
              widen_codes4(lds4(at_sub + row * kRowBytes + i * 16 + q4 * 4), x);
              step(2 * i, x[0], x[1]);
              step(2 * i + 1, x[2], x[3]);
            }
            // powers of two of the keys 2 q4 and 2 q4 + 1, block by block
            float k_power[2 * kBlocks];
            const uint32_t at_exps = exps + (s * 16 + 8 * t + 2 * q4) * kExps;
#pragma unroll
            for (int i = 0; i < kBlocks / 2; ++i) power_word(lds4(at_exps + 4 * i), *reinterpret_cast<float (*)[4]>(&k_power[4 * i]));
#pragma unroll
            for (int e = 0; e < 2 * kHalves; ++e) {
              float x = c_block[0][e] * row_scale[e >> 1] * k_power[(e & 1) * kBlocks];
#pragma unroll
              for (int b = 1; b < kBlocks; ++b) x = fmaf(c_block[b][e] * row_scale[e >> 1], k_power[(e & 1) * kBlocks + b], x);
              sc[s][t][e] = x;
            }
          } else {
#pragma unroll
            for (int i = 0; i < kHd / 32; ++i) {
              const uint4 x = lds16(at_sub + (i >> 1) * 2048 + row * 128 + (((i & 1) * 4 + q4) ^ (row & 7)) * 16);
              step(2 * i, x.x, x.y);
              step(2 * i + 1, x.z, x.w);
            }
          }
          if constexpr (!kFour) {
#pragma unroll
            for (int e = 0; e < 4; ++e) sc[s][t][e] = c_block[0][e];
          }
        }
      // in base-2 units; the reference of a row moves only when a score lies above it
      float most[2] = {-INFINITY, -INFINITY};
#pragma unroll
      for (int s = 0; s < kSubs; ++s)
#pragma unroll
        for (int t = 0; t < 2; ++t) {
          [[maybe_unused]] float k_scale[2] = {1.0f, 1.0f};
          if constexpr (kNarrow) power_pair(exps + s * 16 + 8 * t + 2 * q4, k_scale);
#pragma unroll
          for (int e = 0; e < 2 * kHalves; ++e) {
            float x = sc[s][t][e];
            if constexpr (!kFour) x *= row_scale[e >> 1];
            if constexpr (kNarrow) x *= k_scale[e & 1];
            if (edge && key + 16 * s + 8 * t + 2 * q4 + (e & 1) >= seen[e >> 1]) x = -INFINITY;
            sc[s][t][e] = x;
            most[e >> 1] = fmaxf(most[e >> 1], x);
          }
        }
      if (__builtin_expect(__any_sync(0xffffffffu, most[0] > limit[0] || (!kHalf && most[1] > limit[1])), 0)) {
#pragma unroll
        for (int half = 0; half < kHalves; ++half) {
          float m = most[half];
          m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, 1));
          m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, 2));
          if (m > limit[half]) {
            const bool first = limit[half] == -INFINITY;
            const float apart = m + kFewAbove - ref[half];
            float factor = first ? 0.0f : fast_exp2(-apart);
            ref[half] = limit[half] = m + kFewAbove;
            sum[half] *= factor;
            if constexpr (kNarrow) {  // what was the largest weight may be next to nothing now
              const int k = exponent_of(to[half]), next = min(k + (int)fminf(apart, 512.0f), kFewMostShift);
              if (!first) {
                factor = fast_exp2((float)(next - k) - apart);
                to[half] = power_of_two(next);
              }
            }
#pragma unroll
            for (int i = 0; i < Shape::kOutTiles; ++i) o[i][2 * half] *= factor, o[i][2 * half + 1] *= factor;
          }
        }
      }
      // probabilities, and the weights that the values get
      uint32_t p[kSubs][2][kHalves];
      if constexpr (kNarrow) {
        float heaviest[2] = {0.0f, 0.0f};
#pragma unroll
        for (int s = 0; s < kSubs; ++s)
#pragma unroll
          for (int t = 0; t < 2; ++t) {
            float v_power[2];
            power_pair(exps + (kSubs + s) * 16 + 8 * t + 2 * q4, v_power);
#pragma unroll
            for (int e = 0; e < 2 * kHalves; ++e) {
              const float a = fast_exp2(sc[s][t][e] - ref[e >> 1]);
              sum[e >> 1] += a;
              float weight = a * v_power[e & 1];
              // what is not seen has no weight, whatever it holds
              if (edge && key + 16 * s + 8 * t + 2 * q4 + (e & 1) >= seen[e >> 1]) weight = 0.0f;
              sc[s][t][e] = weight;
              heaviest[e >> 1] = fmaxf(heaviest[e >> 1], weight);
            }
          }
        if (__any_sync(0xffffffffu, heaviest[0] * to[0] > kFewMostWeight || (!kHalf && heaviest[1] * to[1] > kFewMostWeight))) {
#pragma unroll
          for (int half = 0; half < kHalves; ++half) {
            float m = 0.0f;
#pragma unroll
            for (int s = 0; s < kSubs; ++s)
#pragma unroll
              for (int t = 0; t < 2; ++t)
#pragma unroll
                for (int e = 2 * half; e < 2 * half + 2; ++e)
                  if (sc[s][t][e] < INFINITY) m = fmaxf(m, sc[s][t][e]);
            m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, 1));
            m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, 2));
            if (m * to[half] > kFewMostWeight) {
              const int next = kFewWeight - exponent_of(m);
              const float factor = fast_exp2((float)(next - exponent_of(to[half])));
              to[half] = power_of_two(next);
#pragma unroll
              for (int i = 0; i < Shape::kOutTiles; ++i) o[i][2 * half] *= factor, o[i][2 * half + 1] *= factor;
            }
          }
        }
      }
#pragma unroll
      for (int s = 0; s < kSubs; ++s)
#pragma unroll
        for (int t = 0; t < 2; ++t)
#pragma unroll
          for (int half = 0; half < kHalves; ++half) {
            if constexpr (kNarrow) {
              p[s][t][half] = pack_f16(sc[s][t][2 * half] * to[half], sc[s][t][2 * half + 1] * to[half]);
            } else {
              // operands of the second product, each off by up to 2^-8; the sum is that of the rounded ones, so what the rounding
              // changes is how much a key weighs among the others and not the whole row's size
              p[s][t][half] = pack_bf16(fast_exp2(sc[s][t][2 * half] - ref[half]), fast_exp2(sc[s][t][2 * half + 1] - ref[half]));
              sum[half] += bf16_lo(p[s][t][half]) + bf16_hi(p[s][t][half]);
            }
          }
      // output
      constexpr int kLoads = kNarrow ? 1 : kHd / 64, kWords = kNarrow && kHd == 64 ? 2 : 4;
      [[maybe_unused]] uint32_t v_bytes[kSubs][2];  // exponents of the operand's two halves, a key's in either half of a word
      if constexpr (kFour) {
        uint32_t apart = 0;
#pragma unroll
        for (int s = 0; s < kSubs; ++s) {
          const uint32_t at_exps = exps + ((kSubs + s) * 16 + 2 * q4) * kExps, block = g * kExps / 8;
#pragma unroll
          for (int h = 0; h < 2; ++h) {
            if constexpr (kExps == 2) {
              v_bytes[s][h] = __byte_perm(lds4(at_exps + 8 * h * kExps), 0u, 0x4240u + block * 0x101u);
            } else {
              const uint2 x = lds8(at_exps + 8 * h * kExps);
              v_bytes[s][h] = __byte_perm(x.x, x.y, 0x0400u + block * 0x101u) & 0x00ff00ffu;
            }
            apart |= v_bytes[s][h] + 0x007f007fu;
          }
        }
        // (One question for a stage, and what seldom happens out of the way: all that is in line here is too much for the instruction caches as it
        // is, 204 -> 197 us.)  Blocks whose factor is one bf16 number (and so none that are not finite): two keys' codes of a channel are widened together, into a
        // pair of the operand.
        if (__builtin_expect(!__any_sync(0xffffffffu, (apart & 0x01000100u) != 0u), 1)) {
#pragma unroll
          for (int s = 0; s < kSubs; ++s) {
            const uint32_t at_sub = base + (kSubs + s) * Shape::kSubBytes;
            const uint32_t factors[2] = {v_bytes[s][0] + 0x007e007eu << 7, v_bytes[s][1] + 0x007e007eu << 7};
#pragma unroll
            for (int i = 0; i < kLoads; ++i) {
              uint32_t even[2][4], odd[2][4];  // of the even and the odd channels
#pragma unroll
              for (int h = 0; h < 2; ++h) {
                const uint32_t at_row = at_sub + (2 * q4 + 8 * h) * kRowBytes + g * (kRowBytes / 8) + 4 * i;
                const uint32_t a = lds4(at_row), b = lds4(at_row + kRowBytes);
                kv4_widen_by(kv4_low(a), kv4_low(b), factors[h], even[h]);
                kv4_widen_by(kv4_high(a), kv4_high(b), factors[h], odd[h]);
              }
#pragma unroll
              for (int j = 0; j < 8; ++j) {
                const uint32_t b0 = j & 1 ? odd[0][j / 2] : even[0][j / 2], b1 = j & 1 ? odd[1][j / 2] : even[1][j / 2];
                float (&c)[4] = *reinterpret_cast<float (*)[4]>(&o[i * 8 + j][0]);
                mma_16816<false>(c, p[s][0][0], kHalf ? 0u : p[s][0][kHalves - 1], p[s][1][0], kHalf ? 0u : p[s][1][kHalves - 1], b0, b1);
              }
            }
          }
          return;
        }
      }
#pragma unroll
      for (int s = 0; s < kSubs; ++s) {
        const int left = piece.key1 - (key + 16 * s);  // keys of the sub-step that the piece holds
        const uint32_t at_sub = base + (kSubs + s) * Shape::kSubBytes;
#pragma unroll
        for (int i = 0; i < kLoads; ++i) {
          uint32_t v[4][kWords];
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            const int row = 2 * q4 + (e & 1) + 8 * (e >> 1);
            if constexpr (kFour) {
              kv4_widen(lds4(at_sub + row * kRowBytes + g * (kRowBytes / 8) + 4 * i), v_bytes[s][e >> 1] >> 16 * (e & 1) & 0xffu, v[e]);
            } else if constexpr (kWords == 2) {
              const uint2 x = lds8(at_sub + row * 64 + g * 8);
              v[e][0] = x.x, v[e][1] = x.y;
            } else {
              const uint4 x = lds16(kNarrow ? at_sub + row * kHd + g * 16 : at_sub + i * 2048 + row * 128 + (g ^ (row & 7)) * 16);
              v[e][0] = x.x, v[e][1] = x.y, v[e][2] = x.z, v[e][3] = x.w;
            }
            if (left < 16 && row >= left) {  // what lies behind the piece may be anything
#pragma unroll
              for (int j = 0; j < kWords; ++j) v[e][j] = 0u;
            }
          }
#pragma unroll
          for (int j = 0; j < kWords; ++j) {
            constexpr int kPer = kNarrow ? 4 : 2;  // channels of a word
            uint32_t b[kPer][2];
#pragma unroll
            for (int h = 0; h < 2; ++h) {
              const uint32_t lo = __byte_perm(v[2 * h][j], v[2 * h + 1][j], kNarrow ? 0x5140 : 0x5410);
              const uint32_t hi = __byte_perm(v[2 * h][j], v[2 * h + 1][j], kNarrow ? 0x7362 : 0x7632);
              if constexpr (kNarrow) {
                b[0][h] = widen_low(lo), b[1][h] = widen_high(lo), b[kPer - 2][h] = widen_low(hi), b[kPer - 1][h] = widen_high(hi);
              } else {
                b[0][h] = lo, b[1][h] = hi;
              }
            }
#pragma unroll
            for (int n = 0; n < kPer; ++n) {
              const int tile = (i * kWords + j) * kPer + n;
              if (!kNarrow && edge) {
                // A value that is not finite, of a key that some rows see and others do not: a probability of zero would not
                // keep it out.  It is left out of the product and added where it is seen.
                uint32_t b0 = b[n][0], b1 = b[n][1];
                const bool bad = (b0 & 0x7f80u) == 0x7f80u || (b0 & 0x7f800000u) == 0x7f800000u || (b1 & 0x7f80u) == 0x7f80u ||
                                 (b1 & 0x7f800000u) == 0x7f800000u;
                if (__any_sync(0xffffffffu, bad)) {
#pragma unroll 1
                  for (int from = 0; from < 32; ++from) {
                    const uint32_t x0 = __shfl_sync(0xffffffffu, b0, from), x1 = __shfl_sync(0xffffffffu, b1, from);
                    if (q4 != from >> 3) continue;  // the lane holds other channels
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                      const uint32_t x = e < 2 ? x0 : x1, bits = e & 1 ? x >> 16 : x & 0xffffu;
                      if ((bits & 0x7f80u) != 0x7f80u) continue;
                      const float value = __uint_as_float(bits << 16);
                      const int at_key = key + 16 * s + 2 * (from & 3) + (e & 1) + 8 * (e >> 1);
                      // (selects: an accumulator is a register of a fixed name)
                      const bool odd = (from >> 2 & 1) != 0;
#pragma unroll
                      for (int half = 0; half < kHalves; ++half)
                        if (at_key < seen[half]) o[tile][2 * half] += odd ? 0.0f : value, o[tile][2 * half + 1] += odd ? value : 0.0f;
                    }
                  }
                  __syncwarp();
                  if ((b0 & 0x7f80u) == 0x7f80u) b0 &= 0xffff0000u;
                  if ((b0 & 0x7f800000u) == 0x7f800000u) b0 &= 0x0000ffffu;
                  if ((b1 & 0x7f80u) == 0x7f80u) b1 &= 0xffff0000u;
                  if ((b1 & 0x7f800000u) == 0x7f800000u) b1 &= 0x0000ffffu;
                  b[n][0] = b0, b[n][1] = b1;
                }
              }
              if constexpr (Shape::kMoves) {
                float c[4] = {o[tile][0], o[tile][1], 0.0f, 0.0f};
                mma_16816<kNarrow>(c, p[s][0][0], 0u, p[s][1][0], 0u, b[n][0], b[n][1]);
                o[tile][0] = c[0], o[tile][1] = c[1];
              } else {
                float (&c)[4] = *reinterpret_cast<float (*)[4]>(&o[tile][0]);
                mma_16816<kNarrow>(c, p[s][0][0], kHalf ? 0u : p[s][0][kHalves - 1], p[s][1][0], kHalf ? 0u : p[s][1][kHalves - 1], b[n][0], b[n][1]);
              }
            }
          }
        }
      }
    };
    for (int key = piece.key0 + warp * kStageKeys; key < piece.key1 && ok; key += kRound) {
      const uint32_t stage = taken % kStages;
      ok = mbar_wait_warp(&full[stage], (taken / kStages) & 1u, ctl);
      if (!ok) break;
      ++taken;
      if (key + kStageKeys > all_see) take(std::true_type{}, key, ring + stage * Shape::kStageBytes);
      else take(std::false_type{}, key, ring + stage * Shape::kStageBytes);
      __syncwarp();  // all lanes have read the stage
      fetch();
    }

    // ---------------------------------------------------------------- the warps meet
    // tile -> channel: lane g of V's reads holds a run of channels, tile n its n-th
    auto channel_of = [&](int tile, int n) {
      constexpr int kRun = kNarrow || kFour ? kHd / 8 : 8;
      return (tile / kRun) * (8 * kRun) + n * kRun + tile % kRun;
    };
#pragma unroll
    for (int half = 0; half < kHalves; ++half) {
      const float v_scale = kNarrow ? power_of_two(-exponent_of(to[half])) : 1.0f;
      float l = sum[half];
      l += __shfl_xor_sync(0xffffffffu, l, 1);
      l += __shfl_xor_sync(0xffffffffu, l, 2);
      const int r = g + 8 * half;
      if (r < piece.rows) {
        float* dst = smem_o + (warp * Shape::kRows + r) * kHd;
#pragma unroll
        for (int i = 0; i < Shape::kOutTiles; ++i) {
          dst[channel_of(i, 2 * q4)] = o[i][2 * half] * v_scale;
          dst[channel_of(i, 2 * q4 + 1)] = o[i][2 * half + 1] * v_scale;
        }
        if (q4 == 0) {
          float* ml = smem_ml + (warp * Shape::kRows + r) * 2;
          ml[0] = limit[half];
          ml[1] = l;
        }
      }
    }
    __syncthreads();
    auto row_of = [&](int r) {
      const int at_row = piece.row0 + r;
      return (size_t)(seq.row0 + at_row / at.group) * at.q_heads + piece.kv_head * at.group + at_row % at.group;
    };
    // What the warps left in shared memory, weighed against each other; the joint reference is the largest of theirs.  One that
    // has met no key has none (-infinity), and weighs nothing.  `out` gets row, channel, output, reference and sum.
    auto meet = [&](auto out) {
      for (int i = threadIdx.x; i < piece.rows * kHd; i += kKvFewWarps * 32) {
        const int r = i / kHd, ch = i % kHd;
        float m = -INFINITY, l = 0.0f, acc = 0.0f;
#pragma unroll
        for (int w = 0; w < kKvFewWarps; ++w) m = fmaxf(m, smem_ml[(w * Shape::kRows + r) * 2]);
        const float m_use = m == -INFINITY ? 0.0f : m;
#pragma unroll
        for (int w = 0; w < kKvFewWarps; ++w) {
          const float mw = smem_ml[(w * Shape::kRows + r) * 2], weight = mw == -INFINITY ? 1.0f : fast_exp2(mw - m_use);
          l += smem_ml[(w * Shape::kRows + r) * 2 + 1] * weight;
          acc += smem_o[(w * Shape::kRows + r) * kHd + ch] * weight;
        }
        out(r, ch, acc, m, l);
      }
    };
    auto finish = [&](int r, int ch, float acc, float l) {
      at.out[row_of(r) * kHd + ch] = __float2bfloat16_rn(seen_by(r) > 0 ? acc / l : 0.0f);
    };
    if (piece.slot < 0) {
      meet([&](int r, int ch, float acc, float m, float l) {
        finish(r, ch, acc, l);
        if (at.lse != nullptr && ch == 0) at.put_lse((long long)row_of(r), seen_by(r) > 0, m == -INFINITY ? 0.0f : m, l);
      });
    } else {
      meet([&](int r, int ch, float acc, float m, float l) {
        const size_t row = (size_t)piece.slot * kKvFewRows + r;
        __stcg(work.rows + row * kHd + ch, acc);
        if (ch == 0) __stcg(reinterpret_cast<float2*>(work.sums) + row, make_float2(m, l));
      });
      // whoever comes last adds the parts up, in their order
      __threadfence();
      __syncthreads();
      if (threadIdx.x == 0) {
        const int before = atomicAdd(work.joins + piece.join, 1);
        flags[1] = before == piece.parts - 1 ? 1u : 0u;
        if (before == piece.parts - 1) work.joins[piece.join] = 0;
      }
      __syncthreads();
      if (flags[1] != 0) {
        __threadfence();
        // first what every part weighs, [row][part], and the rows' sums behind them; then the rows
        const float2* ml = reinterpret_cast<const float2*>(work.sums) + (size_t)piece.first_slot * kKvFewRows;
        const float* parts = work.rows + (size_t)piece.first_slot * kKvFewRows * kHd;
        const int n = piece.parts;
        for (int r = warp; r < piece.rows; r += kKvFewWarps) {
          float m = -INFINITY, l = 0.0f;
          for (int w = lane; w < n; w += 32) m = fmaxf(m, __ldcg(ml + (size_t)w * kKvFewRows + r).x);
#pragma unroll
          for (int d = 1; d < 32; d *= 2) m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, d));
          const float m_use = m == -INFINITY ? 0.0f : m;
          for (int w = lane; w < n; w += 32) {
            const float2 x = __ldcg(ml + (size_t)w * kKvFewRows + r);
            const float weight = x.x == -INFINITY ? 1.0f : fast_exp2(x.x - m_use);
            smem_o[r * n + w] = weight;
            l += x.y * weight;
          }
#pragma unroll
          for (int d = 1; d < 32; d *= 2) l += __shfl_xor_sync(0xffffffffu, l, d);
          if (lane == 0) {
            smem_ml[r] = l;
            if (at.lse != nullptr) at.put_lse((long long)row_of(r), seen_by(r) > 0, m_use, l);
          }
        }
        __syncthreads();
#pragma unroll 2
        for (int i = threadIdx.x; i < piece.rows * kHd; i += kKvFewWarps * 32) {
          const int r = i / kHd;
          float acc = 0.0f;
#pragma unroll 8
          for (int w = 0; w < n; ++w) acc += __ldcg(parts + (size_t)w * kKvFewRows * kHd + i) * smem_o[r * n + w];
          finish(r, i % kHd, acc, smem_ml[r]);
        }
      }
    }
    __syncthreads();  // the next piece writes where this one was read
  }
  // every load has landed before the CTA may go (all have been waited for, unless a wait was given up)
  for (; taken < fetched; ++taken) {
    const long long t0 = clock64();
    while (!mbar_try_wait(&full[taken % kStages], (taken / kStages) & 1u)) {
      if (clock64() - t0 > kTimeoutCycles) { atomicOr(status, kStatusTimeout); break; }
    }
  }
}

template <int kHd, int kKind, bool kHalf, bool kLong = false>
cudaError_t start(const litevggt_kv_cache& c, const litevggt_kv_batch& b, const KvAttend& a, cudaStream_t s) {
  using Shape = FewShape<kHd, kKind, kHalf, kLong>;
  static_assert(Shape::kCtas * (Shape::kSmemBytes + 1024) <= 228 * 1024, "");
  auto kernel = kv_attn_few_kernel<kHd, kKind, kHalf, kLong>;
  static std::atomic<unsigned long long> done{0};
  const cudaError_t e = set_max_dynamic_smem_once(reinterpret_cast<const void*>(kernel), Shape::kSmemBytes, done);
  if (e != cudaSuccess) return e;
  const KvLaunch work = kv_launch(b, b.few, b.at_few);
  return launch(kernel, dim3((unsigned)work.workers), kKvFewWarps * 32, (size_t)Shape::kSmemBytes, s, c.k_map16, c.v_map16, c.pool,
                kv_arrays(b), work, a, c.status);
}

}  // namespace

int kv_few_ctas(int head_dim, bool narrow) {
  static_assert(FewShape<64, LITEVGGT_KV_E4M3, true>::kCtas == FewShape<64, LITEVGGT_KV_E2M1, true>::kCtas, "");
  return narrow && head_dim == 64 ? FewShape<64, LITEVGGT_KV_E4M3, true>::kCtas : 1;
}

cudaError_t launch_kv_attn_few(const litevggt_kv_cache& c, const litevggt_kv_batch& b, const KvAttend& a, cudaStream_t s, int* launches) {
  const bool half = b.few_rows <= 8, wide = c.cfg.head_dim == 128;
  cudaError_t e;
  auto kinds = [&](auto kind) {
    constexpr int kKind = decltype(kind)::value;
    if constexpr (kKind == LITEVGGT_KV_E2M1) {
      if (half && b.few_keys >= kFewLongPiece) {
        e = wide ? start<128, kKind, true, true>(c, b, a, s) : start<64, kKind, true, true>(c, b, a, s);
        return;
      }
    }
    if (wide) e = half ? start<128, kKind, true>(c, b, a, s) : start<128, kKind, false>(c, b, a, s);
    else e = half ? start<64, kKind, true>(c, b, a, s) : start<64, kKind, false>(c, b, a, s);
  };
  if (c.cfg.dtype == LITEVGGT_KV_E2M1) kinds(std::integral_constant<int, LITEVGGT_KV_E2M1>{});
  else if (c.cfg.dtype == LITEVGGT_KV_E4M3) kinds(std::integral_constant<int, LITEVGGT_KV_E4M3>{});
  else kinds(std::integral_constant<int, LITEVGGT_KV_BF16>{});
  ++*launches;
  return e;
}

}  // namespace lv
