// Rotary positions of several axes: which channels turn together, by what, and how a launch goes over them.  Host arithmetic only.
#pragma once

#include <math.h>
#include <stdint.h>

#include "host_common.h"

namespace lv {

constexpr uint32_t kRotaryMagic = 0x4c56524fu;
constexpr int kRotaryAxes = 4;
constexpr int kRotaryMaxDim = 256;
constexpr int kRotaryPlanes = kRotaryMaxDim / 2;
constexpr int kRotaryThreads = 256;

// A plane is two channels of a head that turn together.  Numbered axis by axis; `turn` is what one step of position turns it by, in
// turns times 2^64: position * turn modulo 2^64 is the angle, wrapped exactly, however far the position is.
struct alignas(16) RotaryTable {
  unsigned long long turn[kRotaryPlanes];
  uint8_t axis[kRotaryPlanes], first[kRotaryPlanes], second[kRotaryPlanes];
  int planes, head_dim;  // channels from 2 * planes on stay as they are
};

static_assert(sizeof(RotaryTable) <= LITEVGGT_ROTARY_BYTES, "");

// One of a launch's tensors.
struct RotaryRows {
  const uint8_t* in;
  uint8_t* out;
  long long in_row, in_head, out_row, out_head;  // bytes
};

struct RotaryLaunch {
  const RotaryTable* table;  // on the device
  RotaryRows rows[2];
  const int* positions;
  long long position_axis, position_row;  // elements
  long long n_rows;
  int heads0, heads;  // of the first tensor, of both
  int planes;         // of a head
  int units, turned;  // of a head, and how many of them turn; the others are copied
  int slots;          // threads that share a unit's heads in a row, of one block
  int all_slots;      // and of all blocks of the row
  int block_rows;
  float sign;
};

inline bool rotary_table(const litevggt_rotary_config& cfg, RotaryTable* t) {
  if (cfg.head_dim < 2 || cfg.head_dim > kRotaryMaxDim || cfg.n_axes < 1 || cfg.n_axes > kRotaryAxes) return false;
  if (cfg.layout != LITEVGGT_ROTARY_HALVES && cfg.layout != LITEVGGT_ROTARY_PAIRS && cfg.layout != LITEVGGT_ROTARY_ACROSS) return false;
  long long width = 0;
  for (int a = 0; a < cfg.n_axes; ++a) {
    if (cfg.sections[a] < 0 || cfg.sections[a] % 2 != 0) return false;
    if (!(cfg.bases[a] > 1.0) || !(cfg.bases[a] < 1e300)) return false;
    width += cfg.sections[a];
  }
  if (width < 2 || width > cfg.head_dim) return false;
  const int all = (int)width / 2;
  const long double two_pi = 6.283185307179586476925286766559005768L;
  int p = 0, at = 0;
  for (int a = 0; a < cfg.n_axes; ++a) {
    const int n = cfg.sections[a] / 2;
    for (int i = 0; i < n; ++i, ++p) {
      const bool across = cfg.layout == LITEVGGT_ROTARY_ACROSS, pairs = cfg.layout == LITEVGGT_ROTARY_PAIRS;
      t->first[p] = (uint8_t)(across ? p : pairs ? at + 2 * i : at + i);
      t->second[p] = (uint8_t)(across ? all + p : pairs ? at + 2 * i + 1 : at + n + i);
      t->axis[p] = (uint8_t)a;
      const long double share = across ? (long double)p / all : (long double)i / n;
      t->turn[p] = (unsigned long long)roundl(ldexpl(expl(-share * logl((long double)cfg.bases[a])) / two_pi, 64));
    }
    at += cfg.sections[a];
  }
  t->planes = p;
  t->head_dim = cfg.head_dim;
  return true;
}

// Whether a unit may be accesses of `v` channels at a time: a unit's planes then have their first channels side by side, and their second
// ones likewise (or, with neighbours as planes, all of them in one access).
inline bool rotary_fits(const RotaryTable& t, bool neighbours, int v) {
  if (t.head_dim % v != 0 || 2 * t.planes % v != 0) return false;
  if (neighbours && v > 1) return true;
  if (t.planes % v != 0) return false;
  for (int p = 0; p < t.planes; ++p) {
    const int p0 = p - p % v;
    if (t.first[p0] % v != 0 || t.second[p0] % v != 0 || t.first[p] != t.first[p0] + p - p0 || t.second[p] != t.second[p0] + p - p0) return false;
  }
  return true;
}

// Bytes from the first to behind the last of a tensor's elements, and whether two such tensors share any.
struct RotarySpan {
  uintptr_t begin;
  unsigned long long row, head, rows, heads, bytes;  // strides and counts; bytes of a head's row
  unsigned long long of_row() const { return (heads - 1) * head + bytes; }
  unsigned long long of_head() const { return (rows - 1) * row + bytes; }
  unsigned long long of_all() const { return (rows - 1) * row + of_row(); }
};
inline bool rotary_same(const RotarySpan& a, const RotarySpan& b) {
  return a.begin == b.begin && (a.row == b.row || a.rows == 1) && (a.head == b.head || a.heads == 1) && a.rows == b.rows && a.heads == b.heads;
}
// Pieces of `of_a` bytes and of `of_b` bytes, one of each in every `period`: whether they are apart.
inline bool rotary_alternate(uintptr_t a, unsigned long long of_a, uintptr_t b, unsigned long long of_b, unsigned long long period) {
  if (of_a > period || of_b > period) return false;
  const unsigned long long ahead = b >= a ? (b - a) % period : (period - (a - b) % period) % period;
  return ahead >= of_a && ahead + of_b <= period;
}
// May answer yes for tensors that interleave in ways other than as columns of one matrix, row by row or head by head.
inline bool rotary_may_meet(const RotarySpan& a, const RotarySpan& b) {
  if (a.begin + a.of_all() <= b.begin || b.begin + b.of_all() <= a.begin) return false;
  if (a.rows > 1 && b.rows > 1 && a.row == b.row && rotary_alternate(a.begin, a.of_row(), b.begin, b.of_row(), a.row)) return false;
  const unsigned long long head = a.heads > 1 ? a.head : b.head;
  const bool heads = (a.heads > 1 || b.heads > 1) && (a.heads == 1 || a.head == head) && (b.heads == 1 || b.head == head);
  return !(heads && rotary_alternate(a.begin, a.of_head(), b.begin, b.of_head(), head));
}
// Whether no two elements of it lie on one another.
inline bool rotary_apart(const RotarySpan& a) {
  const bool heads_in_row = (a.heads == 1 || a.head >= a.bytes) && (a.rows == 1 || a.row >= a.of_row());
  const bool rows_in_head = (a.rows == 1 || a.row >= a.bytes) && (a.heads == 1 || a.head >= (a.rows - 1) * a.row + a.bytes);
  return heads_in_row || rows_in_head;
}

// rotary.cu
cudaError_t launch_rotary(const RotaryLaunch& l, int dtype, int width, bool neighbours, dim3 grid, unsigned threads, cudaStream_t s);

}  // namespace lv

struct litevggt_rotary {
  uint32_t magic;
  int device, num_sms, n_axes;
  bool neighbours;
  lv::RotaryTable table;
  lv::RotaryTable* on_device;  // the caller's
};
