// Stand-ins for the launchers of tallies and eviction, beside kv_host_fakes.cpp.
#include "../paper_2512_04939_b200/csrc/kv_cache.h"

namespace lv {
static int g_weighs = 0, g_evicts = 0;
cudaError_t launch_kv_weigh_few(const litevggt_kv_cache&, const litevggt_kv_batch& b, const KvWeighing&, cudaStream_t, int* n) {
  if (b.weigh.few_at.back() > 0) ++g_weighs, ++*n;
  return cudaSuccess;
}
cudaError_t launch_kv_weigh_tiles(const litevggt_kv_cache&, const litevggt_kv_batch& b, const KvWeighing&, cudaStream_t, int* n) {
  if (b.weigh.items > 0) ++g_weighs, ++*n;
  return cudaSuccess;
}
cudaError_t launch_kv_evict(const litevggt_kv_cache&, const litevggt_kv_batch&, const litevggt_kv_batch&, int, int, int*, cudaStream_t, int* n) {
  ++g_evicts;
  *n += 2;
  return cudaSuccess;
}
}  // namespace lv

extern "C" {
int fake_weighs() { return lv::g_weighs; }
int fake_evicts() { return lv::g_evicts; }
// parts, keys of an item, items, units of few rows of a head; the batch's arrays
void fake_weigh_plan(const litevggt_kv_batch* b, long long* out) {
  out[0] = b->weigh.parts, out[1] = b->weigh.key_block, out[2] = b->weigh.items, out[3] = b->weigh.few_at.back();
  out[4] = (long long)b->o_few_at, out[5] = (long long)b->o_tiles_at, out[6] = (long long)b->o_weigh_joins, out[7] = (long long)b->o_weigh_sums;
  out[8] = (long long)b->bytes, out[9] = (long long)b->image.size();
}
}
