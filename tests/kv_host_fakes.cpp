// Stand-ins for the CUDA runtime and for the kernel launchers behind the paged K/V cache's entry points (kv_api.cu), so that they can be
// driven without a GPU, as if there were two.  "Device" memory is host memory; what is asked of a stream is noted with the device
// that was the current one: the handle of a default stream names another stream on every device.
#include <string.h>

#include "../paper_2512_04939_b200/csrc/kv_cache.h"

using namespace lv;

static int g_device = 0;
static int g_on[2] = {0, 0};  // stream calls by device
static bool g_capturing = false;
static int g_launches = 0;

extern "C" {
void fake_current_device(int d) { g_device = d; }
int fake_get_device() { return g_device; }
int fake_stream_calls(int d) { return g_on[d]; }
void fake_forget() { g_on[0] = g_on[1] = g_launches = 0; }
void fake_capture(int on) { g_capturing = on != 0; }
int fake_launches() { return g_launches; }

cudaError_t cudaGetDevice(int* d) { *d = g_device; return cudaSuccess; }
cudaError_t cudaSetDevice(int d) { g_device = d; return cudaSuccess; }
cudaError_t cudaGetDeviceCount(int* n) { *n = 2; return cudaSuccess; }
cudaError_t cudaDeviceGetAttribute(int* v, cudaDeviceAttr a, int) {
  *v = a == cudaDevAttrComputeCapabilityMajor ? 10 : 148;
  return cudaSuccess;
}
cudaError_t cudaGetLastError() { return cudaSuccess; }
cudaError_t cudaMemcpyAsync(void* d, const void* s, size_t n, cudaMemcpyKind, cudaStream_t) {
  ++g_on[g_device];
  memcpy(d, s, n);
  return cudaSuccess;
}
cudaError_t cudaMemsetAsync(void* p, int v, size_t n, cudaStream_t) {
  ++g_on[g_device];
  memset(p, v, n);
  return cudaSuccess;
}
cudaError_t cudaStreamSynchronize(cudaStream_t) { ++g_on[g_device]; return cudaSuccess; }
cudaError_t cudaStreamIsCapturing(cudaStream_t, cudaStreamCaptureStatus* s) {
  *s = g_capturing ? cudaStreamCaptureStatusActive : cudaStreamCaptureStatusNone;
  return cudaSuccess;
}
}

namespace lv {
bool resolve_encode_tiled(void** fn) { *fn = reinterpret_cast<void*>(1); return true; }
bool make_tmap_bf16_2d(void*, CUtensorMap*, const void*, uint64_t, uint64_t, uint64_t, uint32_t, uint32_t, bool) { return true; }
int kv_few_ctas(int head_dim, bool narrow) { return narrow && head_dim == 64 ? 2 : 1; }
static cudaError_t ran(int* launches) {
  ++g_on[g_device];
  ++g_launches;
  ++*launches;
  return cudaSuccess;
}
cudaError_t launch_kv_append(const litevggt_kv_cache&, const litevggt_kv_batch&, const __nv_bfloat16*, KvStride, const __nv_bfloat16*, KvStride,
                             cudaStream_t, int* n) { return ran(n); }
cudaError_t launch_kv_gather(const litevggt_kv_cache&, const litevggt_kv_batch&, __nv_bfloat16*, __nv_bfloat16*, cudaStream_t, int* n) { return ran(n); }
cudaError_t launch_kv_attn_few(const litevggt_kv_cache&, const litevggt_kv_batch&, const KvAttend&, cudaStream_t, int* n) { return ran(n); }
cudaError_t launch_kv_attn_tiles(const litevggt_kv_cache&, const litevggt_kv_batch&, const KvAttend&, cudaStream_t, int* n) { return ran(n); }
}  // namespace lv
