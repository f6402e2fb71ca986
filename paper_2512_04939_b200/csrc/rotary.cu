// Rotary positions of several axes, for queries and keys in one launch:
//   y_a = x_a cos t - x_b sin t,   y_b = x_a sin t + x_b cos t,   t = position[axis of the plane] * its frequency
// and, as the map is a rotation, the gradient is the same with -t.
//
// Every byte is read once and written once, so HBM bounds it.  A unit is one or two accesses of up to 16 bytes in a head: the first and
// the second channels of as many planes, or neighbours.  A thread keeps a unit's angles and goes with them over heads of a row,
// four loads under way at a time; their cosines are a tenth of its work at four heads, and half at one.
// Angles: position * frequency / (2 pi) as 64-bit fixed point, where the product's wrap is the wrap of the angle.  32 bits of a turn are
// left of it for any position, where a product in 32-bit floating point has 10 of them at position 2^14; the rest is in 32 bits, with one
// rounding at the end.
//
// 83,280 rows, queries and keys of 16 heads of 64 in bf16: 110 us, 6.2 TB/s (a copy makes 6.46), at 67 % of the issue slots; 10,992 rows of 32 and
// 8 heads of 128 in fp32 72 us, 6.2.  One row: 2.9 us.  That is of axes whose planes come in eights side by side; `halves` of sections (16, 24, 24)
// come in fours, in accesses of 8 bytes: 133 us, 5.1 TB/s, and 137 in place in the columns of a projection (sections (16, 16, 32) 111 either way);
// `pairs` 123.  (One load under way at a time 115 and 79 us, two 111 and 78.  A plane's
// frequency from the launch's parameters instead of a table in memory 150: lanes that ask for different words of those wait in turn.)
#include <cuda_fp16.h>

#include "common.cuh"
#include "rotary.h"

namespace lv {

namespace {

// kV elements at a time, in 32 bits.
template <class T, int kV>
struct Run {
  static constexpr int kBytes = kV * (int)sizeof(T), kWords = kBytes / 4;
  uint32_t w[kWords > 0 ? kWords : 1];
  __device__ __forceinline__ void load(const uint8_t* p) {
    if constexpr (kBytes == 16) {
      const uint4 x = *reinterpret_cast<const uint4*>(p);
      w[0] = x.x, w[1] = x.y, w[2] = x.z, w[3] = x.w;
    } else if constexpr (kBytes == 8) {
      const uint2 x = *reinterpret_cast<const uint2*>(p);
      w[0] = x.x, w[1] = x.y;
    } else if constexpr (kBytes == 4) {
      w[0] = *reinterpret_cast<const uint32_t*>(p);
    } else {
      w[0] = *reinterpret_cast<const uint16_t*>(p);
    }
  }
  __device__ __forceinline__ void store(uint8_t* p) const {
    if constexpr (kBytes == 16) *reinterpret_cast<uint4*>(p) = make_uint4(w[0], w[1], w[2], w[3]);
    else if constexpr (kBytes == 8) *reinterpret_cast<uint2*>(p) = make_uint2(w[0], w[1]);
    else if constexpr (kBytes == 4) *reinterpret_cast<uint32_t*>(p) = w[0];
    else *reinterpret_cast<uint16_t*>(p) = (uint16_t)w[0];
  }
  __device__ __forceinline__ float get(int i) const {
    if constexpr (sizeof(T) == 4) {
      return __uint_as_float(w[i]);
    } else {
      const uint32_t bits = (i & 1 ? w[i / 2] >> 16 : w[i / 2]) & 0xffffu;
      if constexpr (std::is_same<T, __half>::value) return __half2float(__ushort_as_half((unsigned short)bits));
      else return __uint_as_float(bits << 16);
    }
  }
  __device__ __forceinline__ void set(const float (&x)[kV]) {
    if constexpr (sizeof(T) == 4) {
#pragma unroll
      for (int i = 0; i < kV; ++i) w[i] = __float_as_uint(x[i]);
    } else if constexpr (kV == 1) {
      if constexpr (std::is_same<T, __half>::value) w[0] = __half_as_ushort(__float2half_rn(x[0]));
      else w[0] = __bfloat16_as_ushort(__float2bfloat16_rn(x[0]));
    } else {
#pragma unroll
      for (int i = 0; i < kV / 2; ++i) {
        if constexpr (std::is_same<T, __half>::value) {
          const __half2 h = __floats2half2_rn(x[2 * i], x[2 * i + 1]);
          w[i] = *reinterpret_cast<const uint32_t*>(&h);
        } else {
          w[i] = pack_bf16(x[2 * i], x[2 * i + 1]);
        }
      }
    }
  }
};

constexpr int kRotaryAhead = 4;  // heads of a thread whose loads are under way together

template <class T, int kV, bool kNeighbours>
__global__ void __launch_bounds__(kRotaryThreads) rotary_kernel(const __grid_constant__ RotaryLaunch l) {
  constexpr int kPlanes = kNeighbours ? kV / 2 : kV, kSize = (int)sizeof(T);
  const int unit = threadIdx.x % l.units, rest = threadIdx.x / l.units, slot = blockIdx.y * l.slots + rest % l.slots;
  const long long row = (long long)blockIdx.x * l.block_rows + rest / l.slots;
  const bool here = rest / l.slots < l.block_rows && row < l.n_rows, turns = unit < l.turned;
  // (the table was there before whatever kernel is still running)
  const int plane0 = unit * kPlanes;
  int a = (2 * l.planes + (unit - l.turned) * kV) * kSize, b = a;
  unsigned long long turn[kPlanes];
  unsigned long long axes = 0;  // a byte for each plane
  if (turns) {
    a = l.table->first[plane0] * kSize;
    if (!kNeighbours) b = l.table->second[plane0] * kSize;
    const unsigned long long* turns_at = l.table->turn + plane0;
    if constexpr (kPlanes == 1) {
      turn[0] = turns_at[0];
    } else {
#pragma unroll
      for (int i = 0; i < kPlanes; i += 2) {
        const ulonglong2 x = *reinterpret_cast<const ulonglong2*>(turns_at + i);
        turn[i] = x.x, turn[i + 1] = x.y;
      }
    }
    const uint8_t* axes_at = l.table->axis + plane0;
    if constexpr (kPlanes == 8) axes = *reinterpret_cast<const unsigned long long*>(axes_at);
    else if constexpr (kPlanes == 4) axes = *reinterpret_cast<const uint32_t*>(axes_at);
    else if constexpr (kPlanes == 2) axes = *reinterpret_cast<const uint16_t*>(axes_at);
    else axes = *axes_at;
  }
  wait_for_previous_kernel();
  if (!here) return;
  auto head_at = [&](int h, bool out) {
    const bool second = h >= l.heads0;
    const RotaryRows& x = l.rows[second ? 1 : 0];
    const int head = second ? h - l.heads0 : h;
    return out ? x.out + row * x.out_row + head * x.out_head : const_cast<uint8_t*>(x.in) + row * x.in_row + head * x.in_head;
  };
  Run<T, kV> xa[kRotaryAhead], xb[kRotaryAhead];
  auto load = [&](int h0) {
#pragma unroll
    for (int i = 0; i < kRotaryAhead; ++i) {
      const int h = h0 + i * l.all_slots;
      if (h >= l.heads) break;
      const uint8_t* p = head_at(h, false);
      xa[i].load(p + a);
      if (!kNeighbours && turns) xb[i].load(p + b);
    }
  };
  load(slot);
  float cs[kPlanes], sn[kPlanes];
  if (turns) {
#pragma unroll
    for (int i = 0; i < kPlanes; ++i) {
      const int position = l.positions[(long long)(axes >> 8 * i & 0xff) * l.position_axis + row * l.position_row];
      const unsigned long long angle = (unsigned long long)(long long)position * turn[i];
      sincospif((float)(int)(angle >> 32) * 4.656612873077392578125e-10f, &sn[i], &cs[i]);  // half turns: 2^-31 of the upper word
      sn[i] *= l.sign;
    }
  }
  for (int h0 = slot; h0 < l.heads; h0 += kRotaryAhead * l.all_slots) {
    if (h0 != slot) load(h0);
#pragma unroll
    for (int i = 0; i < kRotaryAhead; ++i) {
      const int h = h0 + i * l.all_slots;
      if (h >= l.heads) break;
      uint8_t* p = head_at(h, true);
      if (!turns) {
        xa[i].store(p + a);
        continue;
      }
      float ya[kV], yb[kV];
      if constexpr (kNeighbours) {
#pragma unroll
        for (int e = 0; e < kPlanes; ++e) {
          const float x0 = xa[i].get(2 * e), x1 = xa[i].get(2 * e + 1);
          ya[2 * e] = fmaf(-x1, sn[e], x0 * cs[e]);
          ya[2 * e + 1] = fmaf(x0, sn[e], x1 * cs[e]);
        }
      } else {
#pragma unroll
        for (int e = 0; e < kV; ++e) {
          const float x0 = xa[i].get(e), x1 = xb[i].get(e);
          ya[e] = fmaf(-x1, sn[e], x0 * cs[e]);
          yb[e] = fmaf(x0, sn[e], x1 * cs[e]);
        }
        xb[i].set(yb);
        xb[i].store(p + b);
      }
      xa[i].set(ya);
      xa[i].store(p + a);
    }
  }
}

template <class T>
cudaError_t by_width(const RotaryLaunch& l, int v, bool neighbours, dim3 grid, unsigned threads, cudaStream_t s) {
  auto go = [&](auto kernel) { return launch(kernel, grid, threads, 0, s, l); };
  if constexpr (sizeof(T) == 2)
    if (v == 8) return neighbours ? go(rotary_kernel<T, 8, true>) : go(rotary_kernel<T, 8, false>);
  if (v == 4) return neighbours ? go(rotary_kernel<T, 4, true>) : go(rotary_kernel<T, 4, false>);
  if (v == 2) return neighbours ? go(rotary_kernel<T, 2, true>) : go(rotary_kernel<T, 2, false>);
  return go(rotary_kernel<T, 1, false>);
}

}  // namespace

cudaError_t launch_rotary(const RotaryLaunch& l, int dtype, int width, bool neighbours, dim3 grid, unsigned threads, cudaStream_t s) {
  if (dtype == LITEVGGT_BF16) return by_width<__nv_bfloat16>(l, width, neighbours, grid, threads, s);
  if (dtype == LITEVGGT_FP16) return by_width<__half>(l, width, neighbours, grid, threads, s);
  return by_width<float>(l, width, neighbours, grid, threads, s);
}

}  // namespace lv
