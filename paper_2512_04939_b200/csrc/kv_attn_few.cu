// Attention of few rows over a paged K/V cache: single tokens, drafts of a few, heads that share K and V.
//   o_i = sum_j p_ij v_j / sum_j p_ij,   p_ij = 2^(c q_i k_j - m_i)  for the keys j that row i sees
// A piece is up to 16 rows of one sequence and K/V head (tokens times the query heads that share it) against a range of
// keys.  All that counts is that K and V come from memory once and at its full rate: 4 operations a byte at one row.  A warp takes 16
// (or 32) keys at a time straight from global memory into the fragments of mma.m16n8k16; there is no shared memory and no
// barrier on the way.  Which lane loads which 16 bytes follows from the fragments:
//   S = Q K^T   B holds K[key = lane / 4][channels of lane % 4]: the four lanes of a key take 16 bytes each of its row, and the
//               contraction runs over the channels in the order in which they arrive (Q is loaded in the same order)
//   O = P V     B holds V[keys 2q, 2q + 1, 2q + 8, 2q + 9 with q = lane % 4][channel of lane / 4]: a lane loads 8 (or 16)
//               channels of those four keys and pairs them up with byte permutations; its accumulators' keys in S are the same
//               ones, so P goes from accumulator to operand without leaving the lane
// The warps of a CTA take turns on a piece's keys, each with a softmax reference of its own; they meet once at its end.
#include "exp2.cuh"
#include "kv_cache.h"
#include "kv_quant.cuh"

namespace lv {

namespace {

__device__ __forceinline__ void mma_16816(float (&c)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1) {
  asm volatile(
      "mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
      : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
      : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}
__device__ __forceinline__ uint4 load16(const uint8_t* p) { return __ldg(reinterpret_cast<const uint4*>(p)); }

// The reference may lag this far behind a row's maximum (base-2 units) before the row is scaled anew.
constexpr float kFewSlack = 8.0f;

// One sub-step: 16 keys of K and V as they lie in memory.
template <int kHd, bool kNarrow>
struct FewKeys {
  static constexpr int kKLoads = kHd * (kNarrow ? 1 : 2) / 64;  // of 16 bytes, for each of two keys
  static constexpr int kVLoads = kNarrow ? 1 : kHd / 64;        // of 16 bytes (8 for 64 codes), for each of four keys
  static constexpr int kVWords = kNarrow && kHd == 64 ? 2 : 4;
  uint4 k[2][kKLoads];
  uint32_t v[4][kVLoads][kVWords];
  uint32_t k_exp[kNarrow ? 2 : 1], v_exp[kNarrow ? 4 : 1];
};

template <int kHd, bool kNarrow, bool kHalf>
struct FewShape {
  static constexpr int kSubs = !kNarrow && kHd == 128 ? 1 : 2;  // 16 keys each, of a step
  static constexpr int kStep = 16 * kSubs;
  static constexpr int kRows = kHalf ? 8 : 16;
  static constexpr int kOutTiles = kHd / 8;
  static constexpr int kSmemBytes = kKvFewWarps * kRows * (kHd + 2) * 4;
};

// kHalf: at most eight rows, so the lower half of every row tile is empty and takes no registers.
template <int kHd, bool kNarrow, bool kHalf>
__global__ void __launch_bounds__(kKvFewWarps * 32, kHd == 128 && !kHalf ? 1 : 2)
kv_attn_few_kernel(KvPool pool, KvArrays arrays, KvLaunch work, KvAttend at) {
  using Shape = FewShape<kHd, kNarrow, kHalf>;
  using Keys = FewKeys<kHd, kNarrow>;
  constexpr int kEl = kNarrow ? 1 : 2;  // bytes of an element
  constexpr int kSubs = Shape::kSubs;
  extern __shared__ float smem[];
  __shared__ int last_of_join;
  float* smem_o = smem;                                          // [warp][row][channel]
  float* smem_ml = smem + kKvFewWarps * Shape::kRows * kHd;      // [warp][row]{reference, sum}
  wait_for_previous_kernel();
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int g = lane >> 2, q4 = lane & 3;

  for (int id = work.first[blockIdx.x]; id < work.first[blockIdx.x + 1]; ++id) {
    const KvPiece piece = work.pieces[id];
    const KvSeq seq = arrays.seqs[piece.seq];
    const int* pages = arrays.pages + seq.page0;
    const int last_page = (seq.len - 1) >> pool.page_shift;

    // ---------------------------------------------------------------- rows
    auto q_row = [&](int r) {
      const int at_row = piece.row0 + r;
      return at.q + (seq.row0 + at_row / at.group) * at.q_stride.row + (piece.kv_head * at.group + at_row % at.group) * at.q_stride.head;
    };
    uint32_t qa[kHd / 16][kHalf ? 2 : 4];
    {
      // 16 bytes of a K row hold the channels of two contraction steps of 16 (bf16) or of four (codes)
      constexpr int kRun = 16 / kEl;  // channels of a lane that lie side by side
#pragma unroll
      for (int half = 0; half < (kHalf ? 1 : 2); ++half) {
        const int r = g + 8 * half;
        const bool live = r < piece.rows;
        const __nv_bfloat16* src = q_row(live ? r : 0);
#pragma unroll
        for (int i = 0; i < kHd / (4 * kRun); ++i)
#pragma unroll
          for (int j = 0; j < kRun / 4; ++j) {
            uint2 w = make_uint2(0u, 0u);
            if (live) w = *reinterpret_cast<const uint2*>(src + (i * 4 + q4) * kRun + 4 * j);
            qa[i * (kRun / 4) + j][half] = w.x;
            qa[i * (kRun / 4) + j][(kHalf ? 1 : 2) + half] = w.y;
          }
      }
    }
    auto seen_by = [&](int r) { return kv_seen(seq.len, seq.rows, at.causal_block, (piece.row0 + r) / at.group); };
    const int all_see = seen_by(0);                       // keys before this one are seen by every row
    const int seen0 = min(seen_by(g), piece.key1), seen1 = min(seen_by(g + 8), piece.key1);

    float o[Shape::kOutTiles][kHalf ? 2 : 4];
#pragma unroll
    for (int i = 0; i < Shape::kOutTiles; ++i)
#pragma unroll
      for (int j = 0; j < (kHalf ? 2 : 4); ++j) o[i][j] = 0.0f;
    float top[2] = {-INFINITY, -INFINITY}, ref[2] = {0.0f, 0.0f}, sum[2] = {0.0f, 0.0f};  // ref: top where that is finite yet

    // ---------------------------------------------------------------- loads
    // A sub-step's base: its page's rows, from the one of its first key on.  What lies behind the sequence's end comes from its
    // last page, whose rows exist whatever they hold.
    auto base_of = [&](int key) -> long long {
      const int p = min(key >> pool.page_shift, last_page);
      const long long page = pages[p];
      return (page * pool.kv_heads + piece.kv_head) * pool.page_size + (key & (pool.page_size - 1));
    };
    auto load_k = [&](Keys& d, long long row) {
#pragma unroll
      for (int t = 0; t < 2; ++t) {
        const uint8_t* src = pool.k + (row + g + 8 * t) * (kHd * kEl) + q4 * 16;
#pragma unroll
        for (int i = 0; i < Keys::kKLoads; ++i) d.k[t][i] = load16(src + 64 * i);
        if constexpr (kNarrow) d.k_exp[t] = __ldg(pool.k_exp + row + g + 8 * t);
      }
    };
    auto load_v = [&](Keys& d, long long row) {
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const int key = 2 * q4 + (e & 1) + 8 * (e >> 1);
        const uint8_t* src = pool.v + (row + key) * (kHd * kEl);
#pragma unroll
        for (int i = 0; i < Keys::kVLoads; ++i) {
          if constexpr (Keys::kVWords == 2) {
            const uint2 w = __ldg(reinterpret_cast<const uint2*>(src + g * 8));
            d.v[e][i][0] = w.x, d.v[e][i][1] = w.y;
          } else {
            const uint4 w = load16(src + 128 * i + g * 16);
            d.v[e][i][0] = w.x, d.v[e][i][1] = w.y, d.v[e][i][2] = w.z, d.v[e][i][3] = w.w;
          }
        }
        if constexpr (kNarrow) d.v_exp[e] = __ldg(pool.v_exp + row + key);
      }
    };

    // ---------------------------------------------------------------- sweep
    Keys keys[kSubs];
    int key = piece.key0 + warp * Shape::kStep;
    long long rows[kSubs];
    if (key < piece.key1) {
#pragma unroll
      for (int s = 0; s < kSubs; ++s) {
        rows[s] = base_of(key + 16 * s);
        load_k(keys[s], rows[s]);
      }
#pragma unroll
      for (int s = 0; s < kSubs; ++s) load_v(keys[s], rows[s]);
    }
    for (; key < piece.key1; key += kKvFewWarps * Shape::kStep) {
      const int next = key + kKvFewWarps * Shape::kStep;
      const bool more = next < piece.key1;
      if (more) {
#pragma unroll
        for (int s = 0; s < kSubs; ++s) rows[s] = base_of(next + 16 * s);
      }
      // scores
      float sc[kSubs][2][4];
#pragma unroll
      for (int s = 0; s < kSubs; ++s)
#pragma unroll
        for (int t = 0; t < 2; ++t) {
          float (&c)[4] = sc[s][t];
          c[0] = c[1] = c[2] = c[3] = 0.0f;
          auto step = [&](int n, uint32_t b0, uint32_t b1) {
            if constexpr (kHalf) mma_16816(c, qa[n][0], 0u, qa[n][1], 0u, b0, b1);
            else mma_16816(c, qa[n][0], qa[n][1], qa[n][2], qa[n][3], b0, b1);
          };
#pragma unroll
          for (int i = 0; i < Keys::kKLoads; ++i) {
            const uint32_t w[4] = {keys[s].k[t][i].x, keys[s].k[t][i].y, keys[s].k[t][i].z, keys[s].k[t][i].w};
            if constexpr (kNarrow) {
              const KvFactor f = kv_factor(keys[s].k_exp[t]);
              const uint32_t f1 = f.first * 0x10001u, f2 = f.second * 0x10001u;
              const bool second = kv_needs_second(keys[s].k_exp[t]);
#pragma unroll
              for (int j = 0; j < 4; ++j) {
                uint32_t lo = mul_bf16x2(kv_code_bits(__byte_perm(w[j], 0u, 0x1404)), f1);
                uint32_t hi = mul_bf16x2(kv_code_bits(__byte_perm(w[j], 0u, 0x3424)), f1);
                if (second) lo = mul_bf16x2(lo, f2), hi = mul_bf16x2(hi, f2);
                __syncwarp();
                step(4 * i + j, lo, hi);
              }
            } else {
              step(2 * i, w[0], w[1]);
              step(2 * i + 1, w[2], w[3]);
            }
          }
        }
      if (more) {
#pragma unroll
        for (int s = 0; s < kSubs; ++s) load_k(keys[s], rows[s]);
      }
      // probabilities: the reference of a row moves only when a score lies far above it
      const bool edge = key + Shape::kStep > min(all_see, piece.key1);
      float most[2] = {-INFINITY, -INFINITY};
#pragma unroll
      for (int s = 0; s < kSubs; ++s)
#pragma unroll
        for (int t = 0; t < 2; ++t)
#pragma unroll
          for (int e = 0; e < (kHalf ? 2 : 4); ++e) {
            float x = sc[s][t][e] * at.scale_log2;
            if (edge && key + 16 * s + 8 * t + 2 * q4 + (e & 1) >= (e < 2 ? seen0 : seen1)) x = -INFINITY;
            sc[s][t][e] = x;
            most[e >> 1] = fmaxf(most[e >> 1], x);
          }
      if (__any_sync(0xffffffffu, most[0] > top[0] + kFewSlack || (!kHalf && most[1] > top[1] + kFewSlack))) {
#pragma unroll
        for (int half = 0; half < (kHalf ? 1 : 2); ++half) {
          float m = most[half];
          m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, 1));
          m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, 2));
          if (m > top[half]) {
            const float factor = top[half] == -INFINITY ? 0.0f : fast_exp2(ref[half] - m);
            top[half] = m;
            ref[half] = m;
            sum[half] *= factor;
#pragma unroll
            for (int i = 0; i < Shape::kOutTiles; ++i) o[i][2 * half] *= factor, o[i][2 * half + 1] *= factor;
          }
        }
      }
      uint32_t p[kSubs][2][kHalf ? 1 : 2];
#pragma unroll
      for (int s = 0; s < kSubs; ++s)
#pragma unroll
        for (int t = 0; t < 2; ++t)
#pragma unroll
          for (int half = 0; half < (kHalf ? 1 : 2); ++half) {
            const float a = fast_exp2(sc[s][t][2 * half] - ref[half]), b = fast_exp2(sc[s][t][2 * half + 1] - ref[half]);
            // operands of the second product, each off by up to 2^-8; the sum is that of the rounded ones, so what the rounding
            // changes is how much a key weighs among the others and not the whole row's size
            p[s][t][half] = pack_bf16(a, b);
            sum[half] += bf16_lo(p[s][t][half]) + bf16_hi(p[s][t][half]);
          }
      // output
#pragma unroll
      for (int s = 0; s < kSubs; ++s) {
        const int left = piece.key1 - (key + 16 * s);  // keys of the sub-step that the piece holds
        KvFactor f[4];
        bool second = false;
        if constexpr (kNarrow) {
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            f[e] = kv_factor(keys[s].v_exp[e]);
            second = second || kv_needs_second(keys[s].v_exp[e]);
          }
        }
        // channels 2 j, 2 j + 1 of the lane's run, as two operands of two keys each
#pragma unroll
        for (int i = 0; i < Keys::kVLoads; ++i)
#pragma unroll
          for (int j = 0; j < Keys::kVWords; ++j) {
            constexpr int kPer = kNarrow ? 4 : 2;  // channels of a word
            uint32_t w[4];
#pragma unroll
            for (int e = 0; e < 4; ++e) w[e] = keys[s].v[e][i][j];
            if (left < 16) {  // what lies behind the piece may be anything
#pragma unroll
              for (int e = 0; e < 4; ++e)
                if (2 * q4 + (e & 1) + 8 * (e >> 1) >= left) w[e] = 0u;
            }
#pragma unroll
            for (int n = 0; n < kPer; ++n) {
              uint32_t b0, b1;
              if constexpr (kNarrow) {
                const uint32_t pick = (uint32_t)((4 + n) << 12 | n << 4);  // bytes n of both words to the high byte of each half
                b0 = mul_bf16x2(kv_code_bits(__byte_perm(w[0], w[1], pick)), f[0].first | f[1].first << 16);
                b1 = mul_bf16x2(kv_code_bits(__byte_perm(w[2], w[3], pick)), f[2].first | f[3].first << 16);
                if (second) {
                  b0 = mul_bf16x2(b0, f[0].second | f[1].second << 16);
                  b1 = mul_bf16x2(b1, f[2].second | f[3].second << 16);
                }
                if (left < 16) {
                  // a factor behind the piece may be anything too
                  if (2 * q4 >= left) b0 &= 0xffff0000u;
                  if (2 * q4 + 1 >= left) b0 &= 0x0000ffffu;
                  if (2 * q4 + 8 >= left) b1 &= 0xffff0000u;
                  if (2 * q4 + 9 >= left) b1 &= 0x0000ffffu;
                }
                __syncwarp();
              } else {
                b0 = __byte_perm(w[0], w[1], n == 0 ? 0x5410 : 0x7632);
                b1 = __byte_perm(w[2], w[3], n == 0 ? 0x5410 : 0x7632);
              }
              const int tile = (i * Keys::kVWords + j) * kPer + n;
              if (edge) {
                // A value that is not finite, of a key that some rows see and others do not: a probability of zero would not
                // keep it out.  It is left out of the product and added where it is seen.
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
                      if (at_key < seen0) o[tile][0] += odd ? 0.0f : value, o[tile][1] += odd ? value : 0.0f;
                      if (!kHalf && at_key < seen1) o[tile][kHalf ? 0 : 2] += odd ? 0.0f : value, o[tile][kHalf ? 0 : 3] += odd ? value : 0.0f;
                    }
                  }
                  __syncwarp();
                  if ((b0 & 0x7f80u) == 0x7f80u) b0 &= 0xffff0000u;
                  if ((b0 & 0x7f800000u) == 0x7f800000u) b0 &= 0x0000ffffu;
                  if ((b1 & 0x7f80u) == 0x7f80u) b1 &= 0xffff0000u;
                  if ((b1 & 0x7f800000u) == 0x7f800000u) b1 &= 0x0000ffffu;
                }
              }
              if constexpr (kHalf) {
                float c[4] = {o[tile][0], o[tile][1], 0.0f, 0.0f};
                mma_16816(c, p[s][0][0], 0u, p[s][1][0], 0u, b0, b1);
                o[tile][0] = c[0], o[tile][1] = c[1];
              } else {
                mma_16816(o[tile], p[s][0][0], p[s][0][kHalf ? 0 : 1], p[s][1][0], p[s][1][kHalf ? 0 : 1], b0, b1);
              }
            }
          }
      }
      if (more) {
#pragma unroll
        for (int s = 0; s < kSubs; ++s) load_v(keys[s], rows[s]);
      }
    }

    // ---------------------------------------------------------------- the warps meet
    // tile -> channel: lane g of V's loads holds a run of channels, tile n its n-th
    auto channel_of = [&](int tile, int n) {
      constexpr int kRun = kNarrow ? kHd / 8 : 8;
      return (tile / kRun) * (8 * kRun) + n * kRun + tile % kRun;
    };
#pragma unroll
    for (int half = 0; half < (kHalf ? 1 : 2); ++half) {
      float l = sum[half];
      l += __shfl_xor_sync(0xffffffffu, l, 1);
      l += __shfl_xor_sync(0xffffffffu, l, 2);
      const int r = g + 8 * half;
      if (r < piece.rows) {
        float* dst = smem_o + (warp * Shape::kRows + r) * kHd;
#pragma unroll
        for (int i = 0; i < Shape::kOutTiles; ++i) {
          dst[channel_of(i, 2 * q4)] = o[i][2 * half];
          dst[channel_of(i, 2 * q4 + 1)] = o[i][2 * half + 1];
        }
        if (q4 == 0) {
          float* ml = smem_ml + (warp * Shape::kRows + r) * 2;
          ml[0] = top[half];
          ml[1] = l;
        }
      }
    }
    __syncthreads();
    auto store = [&](int r, int ch, float value) {
      const int at_row = piece.row0 + r;
      const size_t row = (size_t)(seq.row0 + at_row / at.group) * at.q_heads + piece.kv_head * at.group + at_row % at.group;
      at.out[row * kHd + ch] = __float2bfloat16_rn(value);
    };
    // The joint reference of several parts of a row is the largest of theirs; a part without keys has none (-infinity), and
    // weighs nothing.
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
      if (piece.slot < 0) {
        store(r, ch, seen_by(r) > 0 ? acc / l : 0.0f);
      } else {
        const size_t row = (size_t)piece.slot * kKvFewRows + r;
        __stcg(work.rows + row * kHd + ch, acc);
        if (ch == 0) __stcg(reinterpret_cast<float2*>(work.sums) + row, make_float2(m, l));
      }
    }
    if (piece.slot >= 0) {
      // whoever comes last adds the parts up, in their order
      __threadfence();
      __syncthreads();
      if (threadIdx.x == 0) {
        const int before = atomicAdd(work.joins + piece.join, 1);
        last_of_join = before == piece.parts - 1;
        if (last_of_join) work.joins[piece.join] = 0;
      }
      __syncthreads();
      if (last_of_join) {
        __threadfence();
        for (int i = threadIdx.x; i < piece.rows * kHd; i += kKvFewWarps * 32) {
          const int r = i / kHd, ch = i % kHd;
          const float2* ml = reinterpret_cast<const float2*>(work.sums) + (size_t)piece.first_slot * kKvFewRows + r;
          const float* part = work.rows + ((size_t)piece.first_slot * kKvFewRows + r) * kHd + ch;
          float m = -INFINITY, l = 0.0f, acc = 0.0f;
          for (int w = 0; w < piece.parts; ++w) m = fmaxf(m, __ldcg(ml + (size_t)w * kKvFewRows).x);
          const float m_use = m == -INFINITY ? 0.0f : m;
          for (int w = 0; w < piece.parts; ++w) {
            const float2 x = __ldcg(ml + (size_t)w * kKvFewRows);
            const float weight = x.x == -INFINITY ? 1.0f : fast_exp2(x.x - m_use);
            l += x.y * weight;
            acc += __ldcg(part + (size_t)w * kKvFewRows * kHd) * weight;
          }
          store(r, ch, seen_by(r) > 0 ? acc / l : 0.0f);
        }
      }
    }
    __syncthreads();  // the next piece writes where this one was read
  }
}

template <int kHd, bool kNarrow, bool kHalf>
cudaError_t start(const litevggt_kv_cache& c, const litevggt_kv_batch& b, const KvAttend& a, cudaStream_t s) {
  using Shape = FewShape<kHd, kNarrow, kHalf>;
  auto kernel = kv_attn_few_kernel<kHd, kNarrow, kHalf>;
  static std::atomic<unsigned long long> done{0};
  const cudaError_t e = set_max_dynamic_smem_once(reinterpret_cast<const void*>(kernel), Shape::kSmemBytes, done);
  if (e != cudaSuccess) return e;
  const KvLaunch work = kv_launch(b, b.few, b.at_few);
  return launch(kernel, dim3((unsigned)work.workers), kKvFewWarps * 32, (size_t)Shape::kSmemBytes, s, c.pool, kv_arrays(b), work, a);
}

}  // namespace

cudaError_t launch_kv_attn_few(const litevggt_kv_cache& c, const litevggt_kv_batch& b, const KvAttend& a, cudaStream_t s, int* launches) {
  int rows = 0;
  for (const KvPiece& p : b.few.pieces) rows = std::max(rows, p.rows);
  const bool half = rows <= 8, narrow = c.cfg.dtype == LITEVGGT_KV_E4M3, wide = c.cfg.head_dim == 128;
  cudaError_t e;
  if (wide) {
    if (narrow) e = half ? start<128, true, true>(c, b, a, s) : start<128, true, false>(c, b, a, s);
    else e = half ? start<128, false, true>(c, b, a, s) : start<128, false, false>(c, b, a, s);
  } else {
    if (narrow) e = half ? start<64, true, true>(c, b, a, s) : start<64, true, false>(c, b, a, s);
    else e = half ? start<64, false, true>(c, b, a, s) : start<64, false, false>(c, b, a, s);
  }
  ++*launches;
  return e;
}

}  // namespace lv
