// The rotary entry points: the checks of arguments, and how a launch is cut.  Host code only.
#include <new>

#include "rotary.h"

namespace lv {
namespace {

constexpr long long kRotaryStride = 1ll << 40;  // elements
constexpr int kRotaryMostHeads = 16384;         // of a tensor: at 256 units a head, blocks of a row are as many as heads, 65,535 at most

bool rotary_ok(const litevggt_rotary* r) { return r != nullptr && r->magic == kRotaryMagic; }

bool stride_ok(int64_t x) { return x >= 0 && x < kRotaryStride; }

}  // namespace
}  // namespace lv

using namespace lv;

extern "C" {

litevggt_status litevggt_rotary_create(const litevggt_rotary_config* cfg, int device, void* memory, size_t bytes, void* stream, litevggt_rotary** out) {
  if (cfg == nullptr || out == nullptr) return LITEVGGT_ERR_NULL;
  *out = nullptr;
  RotaryTable table{};
  if (!rotary_table(*cfg, &table)) return LITEVGGT_ERR_BAD_CONFIG;
  int count = 0, major = 0, sms = 0;
  if (cudaGetDeviceCount(&count) != cudaSuccess || device < 0 || device >= count) {
    (void)cudaGetLastError();
    return LITEVGGT_ERR_CUDA;
  }
  cudaError_t e = cudaDeviceGetAttribute(&major, cudaDevAttrComputeCapabilityMajor, device);
  if (e == cudaSuccess) e = cudaDeviceGetAttribute(&sms, cudaDevAttrMultiProcessorCount, device);
  if (e != cudaSuccess) return cuda_status(e);
  if (major != 10) return LITEVGGT_ERR_ARCH;
  if (memory == nullptr) return LITEVGGT_ERR_NULL;
  if (bytes < sizeof(RotaryTable)) return LITEVGGT_ERR_SHAPE;
  if (!aligned16(memory)) return LITEVGGT_ERR_ALIGN;
  const OnDevice g(device);
  if (!g.ok) return LITEVGGT_ERR_CUDA;
  // In a capture the copy would be made at every replay, and not now.
  cudaStreamCaptureStatus capture = cudaStreamCaptureStatusNone;
  e = cudaStreamIsCapturing((cudaStream_t)stream, &capture);
  if (e == cudaSuccess && capture != cudaStreamCaptureStatusNone) return LITEVGGT_ERR_CUDA;
  if (e == cudaSuccess) e = cudaMemcpyAsync(memory, &table, sizeof(RotaryTable), cudaMemcpyHostToDevice, (cudaStream_t)stream);
  if (e == cudaSuccess) e = cudaStreamSynchronize((cudaStream_t)stream);  // (whichever stream the first call is on)
  if (e != cudaSuccess) return cuda_status(e);
  litevggt_rotary* r = new (std::nothrow) litevggt_rotary();
  if (r == nullptr) return LITEVGGT_ERR_ALLOC;
  r->magic = kRotaryMagic;
  r->device = device;
  r->num_sms = sms;
  r->n_axes = cfg->n_axes;
  r->neighbours = cfg->layout == LITEVGGT_ROTARY_PAIRS;
  r->table = table;
  r->on_device = static_cast<RotaryTable*>(memory);
  *out = r;
  return LITEVGGT_OK;
}

litevggt_status litevggt_rotary_destroy(litevggt_rotary* rotary) {
  if (rotary == nullptr) return LITEVGGT_OK;
  if (!rotary_ok(rotary)) return LITEVGGT_ERR_NULL;
  rotary->magic = 0;
  delete rotary;
  return LITEVGGT_OK;
}

litevggt_status litevggt_rotary_apply(const litevggt_rotary* rotary, const int32_t* positions, int64_t axis_stride, int64_t row_stride,
                                      int64_t rows, int32_t dtype, int32_t back, const litevggt_rotary_tensor* tensors, int32_t n_tensors,
                                      void* stream) {
  if (!rotary_ok(rotary) || tensors == nullptr) return LITEVGGT_ERR_NULL;
  if (rows < 0 || rows > INT32_MAX || n_tensors < 1 || n_tensors > 2) return LITEVGGT_ERR_SHAPE;
  if (dtype != LITEVGGT_BF16 && dtype != LITEVGGT_FP16 && dtype != LITEVGGT_FP32) return LITEVGGT_ERR_SHAPE;
  if (!stride_ok(axis_stride) || !stride_ok(row_stride)) return LITEVGGT_ERR_SHAPE;
  const RotaryTable& t = rotary->table;
  const int size = dtype == LITEVGGT_FP32 ? 4 : 2;
  RotaryLaunch l{};
  RotarySpan in[2], out[2];
  int heads = 0;
  uintptr_t low = 0;  // bits of all addresses and strides
  bool in_place = true;
  for (int i = 0; i < n_tensors; ++i) {
    const litevggt_rotary_tensor& x = tensors[i];
    if (x.heads < 1 || x.heads > kRotaryMostHeads) return LITEVGGT_ERR_SHAPE;
    if (!stride_ok(x.in_row_stride) || !stride_ok(x.in_head_stride) || !stride_ok(x.out_row_stride) || !stride_ok(x.out_head_stride))
      return LITEVGGT_ERR_SHAPE;
    for (int64_t stride : {x.in_row_stride, x.out_row_stride, row_stride})  // (sums of addresses stay inside 64 bits)
      if (rows > 1 && stride > (1ll << 56) / rows) return LITEVGGT_ERR_SHAPE;
    if (rows > 0 && (x.in == nullptr || x.out == nullptr)) return LITEVGGT_ERR_NULL;
    auto span = [&](const void* p, int64_t row, int64_t head) {
      return RotarySpan{reinterpret_cast<uintptr_t>(p), (unsigned long long)row * size, (unsigned long long)head * size,
                        (unsigned long long)rows, (unsigned long long)x.heads, (unsigned long long)t.head_dim * size};
    };
    in[i] = span(x.in, x.in_row_stride, x.in_head_stride);
    out[i] = span(x.out, x.out_row_stride, x.out_head_stride);
    for (const RotarySpan& s : {in[i], out[i]}) {
      low |= s.begin;
      if (rows > 1) low |= s.row;
      if (x.heads > 1) low |= s.head;
    }
    l.rows[i] = RotaryRows{static_cast<const uint8_t*>(x.in), static_cast<uint8_t*>(x.out), (long long)in[i].row, (long long)in[i].head,
                           (long long)out[i].row, (long long)out[i].head};
    heads += x.heads;
    in_place = in_place && rotary_same(in[i], out[i]);
  }
  if (rows == 0) return LITEVGGT_OK;
  if (positions == nullptr) return LITEVGGT_ERR_NULL;
  if (low % size != 0 || reinterpret_cast<uintptr_t>(positions) % 4 != 0) return LITEVGGT_ERR_ALIGN;
  // A row of a head is read before it is written, by the same thread: that makes turning in place safe, and nothing else.
  const RotarySpan where{reinterpret_cast<uintptr_t>(positions), (unsigned long long)row_stride * 4, (unsigned long long)axis_stride * 4,
                         (unsigned long long)rows, (unsigned long long)rotary->n_axes, 4};
  for (int i = 0; i < n_tensors; ++i) {
    if (!rotary_apart(out[i]) || rotary_may_meet(out[i], where)) return LITEVGGT_ERR_SHAPE;
    for (int j = 0; j < n_tensors; ++j) {
      if (!(i == j && rotary_same(in[i], out[i])) && rotary_may_meet(out[i], in[j])) return LITEVGGT_ERR_SHAPE;
      if (i < j && rotary_may_meet(out[i], out[j])) return LITEVGGT_ERR_SHAPE;
    }
  }
  int v = 16 / size;
  while (v > 1 && (low % (uintptr_t)(v * size) != 0 || !rotary_fits(t, rotary->neighbours, v))) v /= 2;
  const bool neighbours = rotary->neighbours && v > 1;
  l.table = rotary->on_device;
  l.planes = t.planes;
  l.positions = positions;
  l.position_axis = axis_stride;
  l.position_row = row_stride;
  l.n_rows = rows;
  l.heads0 = tensors[0].heads;
  l.heads = heads;
  l.turned = neighbours ? 2 * t.planes / v : t.planes / v;
  l.units = l.turned + (in_place ? 0 : (t.head_dim - 2 * t.planes) / v);
  l.sign = back != 0 ? -1.0f : 1.0f;
  // A unit's heads by so many threads in a row: four heads each share one set of angles where that fills the chip all the same.
  const long long full = (long long)rotary->num_sms * 2048;
  int slots = (heads + 3) / 4;
  if (rows * l.units * slots < full) slots = heads;
  const int across = (slots * l.units + kRotaryThreads - 1) / kRotaryThreads;  // blocks of a row (units are 256 at most)
  l.slots = (slots + across - 1) / across;
  if (l.slots * l.units > kRotaryThreads) l.slots = kRotaryThreads / l.units;
  const int grid_y = (slots + l.slots - 1) / l.slots;
  l.all_slots = l.slots * grid_y;
  l.block_rows = kRotaryThreads / (l.units * l.slots);
  if (l.block_rows > rows) l.block_rows = (int)rows;
  const long long blocks = (rows + l.block_rows - 1) / l.block_rows;
  const unsigned threads = (unsigned)round_up((long long)l.units * l.slots * l.block_rows, 32);
  const OnDevice g(rotary->device);
  if (!g.ok) return LITEVGGT_ERR_CUDA;
  return cuda_status(launch_rotary(l, dtype, v, neighbours, dim3((unsigned)blocks, (unsigned)grid_y), threads, (cudaStream_t)stream));
}

}  // extern "C"
