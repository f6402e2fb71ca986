// The kernels that write the paged K/V cache and read it back.
//
// Writing and reading move every byte once and compute next to nothing, so HBM bounds both.  A unit of work is one
// row of one K/V head, K and V alike: 16 bytes of bf16 a lane, the 8 (or 16) lanes of a row side by side in the warp, so
// that a row's largest magnitude takes three (four) shuffles and its codes leave as 64 (128) bytes in a row.  83,280 rows of 16
// heads of 64: written as bf16 110 us, 6.2 TB/s, as E4M3 85 us, 6.0; read back 106 us, 6.4, and 82 us, 6.3 (a copy makes 6.46).
#include "kv_cache.h"
#include "kv_quant.cuh"

namespace lv {

namespace {

constexpr int kMoveThreads = 256;

// The sequence that a row of the packed tensors belongs to.
__device__ __forceinline__ KvSeq seq_of_row(const KvArrays& a, int row) {
  int lo = 0, hi = a.n_seq - 1;
  while (lo < hi) {  // the last one that begins at or before the row; ones without rows share their successor's start
    const int mid = (lo + hi + 1) >> 1;
    if (a.seqs[mid].row0 <= row) lo = mid;
    else hi = mid - 1;
  }
  return a.seqs[lo];
}
// Index of a row's token and head among the pool's rows, of which there are less than 2^31.
__device__ __forceinline__ unsigned pool_row(const KvPool& pool, const KvArrays& a, int row, int head) {
  const KvSeq q = seq_of_row(a, row);
  const int token = q.len - q.rows + (row - q.row0);
  const unsigned page = (unsigned)a.pages[q.page0 + (token >> pool.page_shift)];
  return ((page * (unsigned)pool.kv_heads + (unsigned)head) << pool.page_shift) + (unsigned)(token & (pool.page_size - 1));
}

// Largest magnitudes of a row of K and of V, as the bits of bf16 numbers in the low and the high half.
__device__ __forceinline__ uint32_t lane_top(const uint4& x) {
  const uint32_t m = __vmaxu2(__vmaxu2(x.x & 0x7fff7fffu, x.y & 0x7fff7fffu), __vmaxu2(x.z & 0x7fff7fffu, x.w & 0x7fff7fffu));
  return __vmaxu2(m, m >> 16);  // (low half)
}
template <int kLanes>
__device__ __forceinline__ uint32_t row_tops(const uint4& k, const uint4& v) {
  uint32_t m = __byte_perm(lane_top(k), lane_top(v), 0x5410);
#pragma unroll
  for (int d = 1; d < kLanes; d *= 2) m = __vmaxu2(m, __shfl_xor_sync(0xffffffffu, m, d));
  return m;
}
__device__ __forceinline__ uint2 row_codes(const uint4& x, uint32_t byte) {
  if (byte == kKvNanByte) return make_uint2(0u, 0u);
  const float f = kv_inverse_scale(byte);
  return make_uint2(pack_e4m3x4(bf16_lo(x.x) * f, bf16_hi(x.x) * f, bf16_lo(x.y) * f, bf16_hi(x.y) * f),
                    pack_e4m3x4(bf16_lo(x.z) * f, bf16_hi(x.z) * f, bf16_lo(x.w) * f, bf16_hi(x.w) * f));
}
// Eight codes to eight bf16.
__device__ __forceinline__ uint4 row_values(const uint2& codes, uint32_t byte) {
  const KvFactor f = kv_factor(byte);
  const uint32_t w[2] = {codes.x, codes.y};
  uint32_t r[4];
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    r[2 * i] = mul_bf16x2(kv_code_bits(__byte_perm(w[i], 0u, 0x1404)), f.first * 0x10001u);
    r[2 * i + 1] = mul_bf16x2(kv_code_bits(__byte_perm(w[i], 0u, 0x3424)), f.first * 0x10001u);
  }
  if (kv_needs_second(byte)) {
#pragma unroll
    for (int i = 0; i < 4; ++i) r[i] = mul_bf16x2(r[i], f.second * 0x10001u);
  }
  return make_uint4(r[0], r[1], r[2], r[3]);
}

// Where a lane's 16 bytes of a unit lie: kUnits of them to a group of lanes, a block's side by side.  (Rows times heads fit 31 bits.)
template <int kHd, int kUnits>
struct MoveUnits {
  static constexpr int kLanes = kHd / 8, kGroups = kMoveThreads / kLanes;
  unsigned first, units;
  int part;
  __device__ __forceinline__ explicit MoveUnits(unsigned n)
      : first(blockIdx.x * (unsigned)(kGroups * kUnits) + threadIdx.x / kLanes), units(n), part(threadIdx.x % kLanes) {}
  __device__ __forceinline__ unsigned unit(int i) const { return first + i * kGroups; }
  __device__ __forceinline__ bool live(int i) const { return unit(i) < units; }
};

template <int kHd, bool kNarrow, int kUnits>
__global__ void __launch_bounds__(kMoveThreads)
kv_append_kernel(KvPool pool, KvArrays arrays, const __nv_bfloat16* __restrict__ k, KvStride ks, const __nv_bfloat16* __restrict__ v,
                 KvStride vs, unsigned units) {
  constexpr int kLanes = kHd / 8;
  wait_for_previous_kernel();
  const MoveUnits<kHd, kUnits> mine(units);
  const int part = mine.part;
  uint4 xk[kUnits], xv[kUnits];
  size_t at[kUnits];
#pragma unroll
  for (int i = 0; i < kUnits; ++i) {
    xk[i] = xv[i] = make_uint4(0u, 0u, 0u, 0u);
    at[i] = 0;
    if (!mine.live(i)) continue;
    const int row = (int)(mine.unit(i) / (unsigned)pool.kv_heads), head = (int)(mine.unit(i) % (unsigned)pool.kv_heads);
    xk[i] = ldg16(k + row * ks.row + head * ks.head + part * 8);
    xv[i] = ldg16(v + row * vs.row + head * vs.head + part * 8);
    at[i] = pool_row(pool, arrays, row, head);
  }
#pragma unroll
  for (int i = 0; i < kUnits; ++i) {
    if constexpr (kNarrow) {
      const uint32_t tops = row_tops<kLanes>(xk[i], xv[i]), bk = kv_exponent_byte(tops & 0xffffu), bv = kv_exponent_byte(tops >> 16);
      if (mine.live(i)) {
        *reinterpret_cast<uint2*>(pool.k + at[i] * kHd + part * 8) = row_codes(xk[i], bk);
        *reinterpret_cast<uint2*>(pool.v + at[i] * kHd + part * 8) = row_codes(xv[i], bv);
        if (part == 0) pool.k_exp[at[i]] = (uint8_t)bk;
        if (part == 1) pool.v_exp[at[i]] = (uint8_t)bv;
      }
    } else if (mine.live(i)) {
      stg16(pool.k + (at[i] * kHd + part * 8) * 2, xk[i]);
      stg16(pool.v + (at[i] * kHd + part * 8) * 2, xv[i]);
    }
  }
}

template <int kHd, bool kNarrow, int kUnits>
__global__ void __launch_bounds__(kMoveThreads)
kv_gather_kernel(KvPool pool, KvArrays arrays, __nv_bfloat16* __restrict__ k, __nv_bfloat16* __restrict__ v, unsigned units) {
  wait_for_previous_kernel();
  const MoveUnits<kHd, kUnits> mine(units);
  const int part = mine.part;
  uint4 xk[kUnits], xv[kUnits];  // as they lie in the pool
  uint32_t bk[kUnits], bv[kUnits];
#pragma unroll
  for (int i = 0; i < kUnits; ++i) {
    if (!mine.live(i)) continue;
    const size_t at = pool_row(pool, arrays, (int)(mine.unit(i) / (unsigned)pool.kv_heads), (int)(mine.unit(i) % (unsigned)pool.kv_heads));
    if constexpr (kNarrow) {
      const uint2 ck = *reinterpret_cast<const uint2*>(pool.k + at * kHd + part * 8);
      const uint2 cv = *reinterpret_cast<const uint2*>(pool.v + at * kHd + part * 8);
      xk[i].x = ck.x, xk[i].y = ck.y, xv[i].x = cv.x, xv[i].y = cv.y;
      bk[i] = pool.k_exp[at];
      bv[i] = pool.v_exp[at];
    } else {
      xk[i] = ldg16(pool.k + (at * kHd + part * 8) * 2);
      xv[i] = ldg16(pool.v + (at * kHd + part * 8) * 2);
    }
  }
#pragma unroll
  for (int i = 0; i < kUnits; ++i) {
    if (!mine.live(i)) continue;
    if constexpr (kNarrow) {
      xk[i] = row_values(make_uint2(xk[i].x, xk[i].y), bk[i]);
      xv[i] = row_values(make_uint2(xv[i].x, xv[i].y), bv[i]);
    }
    stg16(k + (size_t)mine.unit(i) * kHd + part * 8, xk[i]);
    stg16(v + (size_t)mine.unit(i) * kHd + part * 8, xv[i]);
  }
}

// Calls f with the head dimension, the pool's type and the units of a lane group as constants, and the blocks that this takes.
// One unit where all blocks are on the chip at once (1,041 rows of 16 heads in E4M3: 2.9 us written, 2.5 read; two: 3.5 and
// 2.9), two where that keeps more bytes under way (83,280 rows read back: 82.5 us against 95.6; four are no better).
template <class F>
void by_kind(const litevggt_kv_cache& c, long long units, const F& f) {
  using std::integral_constant;
  auto sized = [&](auto hd, auto narrow) {
    const long long per_block = kMoveThreads / (decltype(hd)::value / 8), blocks = (units + per_block - 1) / per_block;
    if (blocks <= (long long)c.num_sms * (2048 / kMoveThreads)) f(hd, narrow, integral_constant<int, 1>{}, (unsigned)blocks);
    else f(hd, narrow, integral_constant<int, 2>{}, (unsigned)((blocks + 1) / 2));
  };
  const bool narrow = c.cfg.dtype == LITEVGGT_KV_E4M3;
  if (c.cfg.head_dim == 64) {
    if (narrow) sized(integral_constant<int, 64>{}, integral_constant<bool, true>{});
    else sized(integral_constant<int, 64>{}, integral_constant<bool, false>{});
  } else {
    if (narrow) sized(integral_constant<int, 128>{}, integral_constant<bool, true>{});
    else sized(integral_constant<int, 128>{}, integral_constant<bool, false>{});
  }
}

}  // namespace

cudaError_t launch_kv_append(const litevggt_kv_cache& c, const litevggt_kv_batch& b, const __nv_bfloat16* k, KvStride k_stride,
                             const __nv_bfloat16* v, KvStride v_stride, cudaStream_t s, int* launches) {
  const long long units = b.rows * c.cfg.kv_heads;
  cudaError_t e = cudaSuccess;
  by_kind(c, units, [&](auto hd, auto narrow, auto per, unsigned blocks) {
    e = launch(kv_append_kernel<decltype(hd)::value, decltype(narrow)::value, decltype(per)::value>, dim3(blocks), kMoveThreads, 0, s, c.pool,
               kv_arrays(b), k, k_stride, v, v_stride, (unsigned)units);
  });
  ++*launches;
  return e;
}

cudaError_t launch_kv_gather(const litevggt_kv_cache& c, const litevggt_kv_batch& b, __nv_bfloat16* k, __nv_bfloat16* v, cudaStream_t s,
                             int* launches) {
  const long long units = b.rows * c.cfg.kv_heads;
  cudaError_t e = cudaSuccess;
  by_kind(c, units, [&](auto hd, auto narrow, auto per, unsigned blocks) {
    e = launch(kv_gather_kernel<decltype(hd)::value, decltype(narrow)::value, decltype(per)::value>, dim3(blocks), kMoveThreads, 0, s, c.pool,
               kv_arrays(b), k, v, (unsigned)units);
  });
  ++*launches;
  return e;
}

}  // namespace lv
