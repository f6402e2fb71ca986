// Stand-ins for the CUDA runtime and the kernel launch behind the rotary entry points (rotary_api.cu): what would be launched is kept.
#include <string.h>

#include "../paper_2512_04939_b200/csrc/rotary.h"

using namespace lv;

static RotaryLaunch g_launch;
static int g_launches = 0, g_width = 0, g_neighbours = 0, g_device = 0, g_launched_on = -1, g_copied_on = -1;
static bool g_capturing = false;
static unsigned g_blocks = 0, g_threads = 0, g_across = 0;

extern "C" {
cudaError_t cudaGetDevice(int* d) { *d = g_device; return cudaSuccess; }
cudaError_t cudaSetDevice(int d) { g_device = d; return cudaSuccess; }
cudaError_t cudaGetDeviceCount(int* n) { *n = 2; return cudaSuccess; }
cudaError_t cudaDeviceGetAttribute(int* v, cudaDeviceAttr a, int) {
  *v = a == cudaDevAttrComputeCapabilityMajor ? 10 : 148;
  return cudaSuccess;
}
cudaError_t cudaGetLastError() { return cudaSuccess; }
cudaError_t cudaMemcpyAsync(void* d, const void* s, size_t n, cudaMemcpyKind, cudaStream_t) {
  g_copied_on = g_device;
  memcpy(d, s, n);
  return cudaSuccess;
}
cudaError_t cudaStreamSynchronize(cudaStream_t) { return cudaSuccess; }
cudaError_t cudaStreamIsCapturing(cudaStream_t, cudaStreamCaptureStatus* s) {
  *s = g_capturing ? cudaStreamCaptureStatusActive : cudaStreamCaptureStatusNone;
  return cudaSuccess;
}
void fake_capture(int on) { g_capturing = on != 0; }
int fake_copied_on() { return g_copied_on; }
int fake_launches() { return g_launches; }
int fake_get_device() { return g_device; }
int fake_launched_on() { return g_launched_on; }
// width, neighbours, units, turned, slots, block_rows, blocks, planes, threads, blocks of a row, slots of a row
void fake_last(int* out) {
  const int x[11] = {g_width, g_neighbours, g_launch.units, g_launch.turned, g_launch.slots, g_launch.block_rows, (int)g_blocks, g_launch.planes,
                     (int)g_threads, (int)g_across, g_launch.all_slots};
  for (int i = 0; i < 11; ++i) out[i] = x[i];
}
void fake_plane(int p, int* first, int* second, int* axis, unsigned long long* turn) {
  *first = g_launch.table->first[p];
  *second = g_launch.table->second[p];
  *axis = g_launch.table->axis[p];
  *turn = g_launch.table->turn[p];
}
}

namespace lv {
cudaError_t launch_rotary(const RotaryLaunch& l, int, int width, bool neighbours, dim3 grid, unsigned threads, cudaStream_t) {
  g_launch = l;
  g_width = width;
  g_neighbours = neighbours;
  g_blocks = grid.x;
  g_across = grid.y;
  g_threads = threads;
  g_launched_on = g_device;
  ++g_launches;
  return cudaSuccess;
}
}  // namespace lv
