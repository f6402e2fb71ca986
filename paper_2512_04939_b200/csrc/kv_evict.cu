// Eviction from the paged K/V cache: every head of every sequence keeps its first and its last tokens and, of the others, those that
// have drawn most of the attention (of equal tallies the earlier), and all of them move to other pages in the order that they were in.
//
// Choosing: one cluster of CTAs for a head of a sequence, each with a run of its tokens.  Tallies become numbers that order as they do,
// in shared memory, and the least one that stays is found digit by digit (11, 11 and 10 bits): a histogram in each CTA, whose bins that
// are not empty are added up in the first CTA's, which looks for the bin.  Then every warp counts what stays of its own tokens and, when all
// counts are known, writes their numbers.  Sums are of whole numbers, so nothing depends on an order.
// Moving: HBM bounds it; 16 bytes of K and of V a lane, a warp's writes side by side in the pages that are filled.
//
// Choosing 131,072 of 520,500 tokens in each of 4 heads: 39.5 us, on the 64 SMs that 4 clusters of 16 are, by the meetings of a cluster and the
// passes over what it holds (260 when each pass read the tallies again); 2,082 of up to 5,205 for 24 sequences of 16 heads 19.6 us; 522 of 1,044
// 7.3 us, of which most is meetings of the block.  Moving the second of these in 8 bits of 128 channels: 52 us, 5.1 TB/s (three and four
// units a lane instead of two: 52, 55); the first 47.7 us, 281 MB, 5.9 TB/s.
#include "kv_cache.h"
#include "kv_quant.cuh"

namespace lv {

namespace {

constexpr int kPickThreads = 512, kPickMostThreads = 1024, kPickBins = 2048;
constexpr int kPickMostBlocks = 16, kPickPortableBlocks = 8;  // of a cluster
constexpr int kPickAhead = 4;                                 // loads of four tallies that a thread has under way together
constexpr int kPickStep = 128;                                // tokens of a warp's step
constexpr uint32_t kPickFew = 512;                            // numbers that are compared with one another
constexpr int kPickMostHeld = 48 * 1024;                      // numbers in a CTA's shared memory; what lies behind them is read again

// Orders as the tallies do; zeros are equal, NaN is less than any number; 0 is nobody's.
__device__ __forceinline__ uint32_t order_of(float x) {
  if (x != x) return 1u;
  const uint32_t bits = __float_as_uint(x + 0.0f);  // -0 + 0 = 0
  return bits & 0x80000000u ? ~bits : bits | 0x80000000u;
}

__device__ __forceinline__ uint32_t ld_cluster(uint32_t addr) {
  uint32_t v;
  asm volatile("ld.shared::cluster.u32 %0, [%1];" : "=r"(v) : "r"(addr) : "memory");
  return v;
}
__device__ __forceinline__ void add_cluster(uint32_t addr, uint32_t n) {
  asm volatile("red.shared::cluster.add.u32 [%0], %1;" ::"r"(addr), "r"(n) : "memory");
}

struct alignas(16) PickShared {
  uint32_t bins[kPickBins];   // of this CTA's tokens
  uint32_t joint[kPickBins];  // of the cluster's, in its first CTA; of a CTA by itself the list of those that are few
  uint32_t warp_sums[kPickMostThreads / 32][2];
  uint32_t counts[2];         // of this CTA: above the least that stays, equal to it
  uint32_t bin, left, in_bin; // first CTA: the bin that the least one lies in, how many of it stay, and are there
  uint32_t listed;
  uint32_t scan[kPickMostThreads / 32];
};

// blockIdx.x = (sequence * heads + head) * blocks of a cluster + block; `held`: numbers that a warp keeps in shared memory
// (three blocks of the smaller kind on an SM: 16 heads of 24 sequences are there at once)
template <int kThreads>
__global__ void __launch_bounds__(kThreads, kThreads == kPickThreads ? 3 : 1)
kv_pick_kernel(KvPool pool, KvArrays from, KvArrays into, int first, int last, int blocks, int held, int* kept) {
  __shared__ PickShared sh;
  extern __shared__ uint4 numbers[];  // [warp][held / 4]
  constexpr int threads = kThreads, n_warps = threads / 32;
  const int rank = blocks > 1 ? (int)cluster_ctarank() : 0, pair = (int)blockIdx.x / blocks;
  const int head = pair % pool.kv_heads, warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  // (a batch's arrays were there before whatever kernel is still running)
  const KvSeq src = from.seqs[pair / pool.kv_heads], dst = into.seqs[pair / pool.kv_heads];
  const int n = src.len, m = dst.len;
  wait_for_previous_kernel();
  int* out = kept + (long long)dst.row0 * pool.kv_heads + head;  // the i-th kept token's number at i * heads
  auto put = [&](int at, int token) { out[(long long)at * pool.kv_heads] = token; };
  const int all = blocks * threads, mine = rank * threads + threadIdx.x;
  if (m >= n) {  // (the same for the whole cluster)
    for (int i = mine; i < m; i += all) put(i, i);
    return;
  }
  for (int i = mine; i < first; i += all) put(i, i);
  for (int i = mine; i < last; i += all) put(m - last + i, n - last + i);
  const int choose = m - first - last;  // of the tokens in between
  if (choose <= 0) return;
  // This warp's run of tokens, in steps of kPickStep, four of each lane: all from the first one that may go on, rounded down to four, which
  // lie side by side in a page.  Those outside the range are nobody's number.
  const int low = first & ~3, span = n - last - low, warps = blocks * n_warps;
  const int run = (int)((((long long)span + warps - 1) / warps + kPickStep - 1) / kPickStep * kPickStep);
  const long long begin64 = (long long)(rank * n_warps + warp) * run;
  const int begin = low + (int)min(begin64, (long long)span), end = low + (int)min(begin64 + run, (long long)span);
  auto tallies_at = [&](int token) {
    const size_t page = (size_t)from.pages[src.page0 + (token >> pool.page_shift)];
    return *reinterpret_cast<const float4*>(pool.weights + ((page * pool.kv_heads + head) << pool.page_shift) + (token & (pool.page_size - 1)));
  };
  auto numbers_of = [&](int token, const float4& x) {
    auto one = [&](int i, float y) { return token + i >= first && token + i < n - last ? order_of(y) : 0u; };
    return make_uint4(one(0, x.x), one(1, x.y), one(2, x.z), one(3, x.w));
  };
  uint4* mine_held = numbers + (warp * held >> 2);
  const int end_held = min(end, begin + held);
  for (int at = begin + 4 * lane; at - 4 * lane < end_held; at += kPickStep * kPickAhead) {
    float4 x[kPickAhead];
#pragma unroll
    for (int j = 0; j < kPickAhead; ++j)
      if (at + kPickStep * j < end_held) x[j] = tallies_at(at + kPickStep * j);
#pragma unroll
    for (int j = 0; j < kPickAhead; ++j)
      if (at + kPickStep * j < end_held) mine_held[(at + kPickStep * j - begin) >> 2] = numbers_of(at + kPickStep * j, x[j]);
  }
  // (a thread reads what it has written itself)
  auto numbers_at = [&](int token) {
    if (token >= end) return make_uint4(0u, 0u, 0u, 0u);
    return token < end_held ? mine_held[(token - begin) >> 2] : numbers_of(token, tallies_at(token));
  };
  auto together = [&]() {
    if (blocks > 1) cluster_sync();
    else __syncthreads();
  };
  const uint32_t joint0 = blocks > 1 ? mapa_u32(smem_u32(sh.joint), 0) : smem_u32(sh.joint);
  const uint32_t* joint = blocks > 1 ? sh.joint : sh.bins;  // in the first CTA

  uint32_t prefix = 0, known = 0, left = (uint32_t)choose;  // the upper bits of the least that stays; their mask; how many of those with them stay
  for (int pass = 0; pass < 3; ++pass) {
    const int shift = pass == 0 ? 21 : pass == 1 ? 10 : 0;
    const uint32_t digits = pass == 2 ? 1023u : 2047u;
    for (int i = threadIdx.x; i < kPickBins; i += threads) {
      sh.bins[i] = 0u;
      if (blocks > 1) sh.joint[i] = 0u;
    }
    together();
    for (int at = begin; at < end; at += kPickStep) {
      const uint4 x4 = numbers_at(at + 4 * lane);
      const uint32_t x[4] = {x4.x, x4.y, x4.z, x4.w};
      bool counts[4], some = false;
      uint32_t bin[4];
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        counts[j] = (x[j] & known) == prefix;
        bin[j] = x[j] >> shift & digits;
        some = some || counts[j];
      }
      if (!__any_sync(0xffffffffu, some)) continue;
      // one of all where they agree, as where no tallies have been taken: the unit that adds takes them one by one
      const uint32_t first_bin = __shfl_sync(0xffffffffu, bin[0], 0);
      bool alike = true;
#pragma unroll
      for (int j = 0; j < 4; ++j) alike = alike && counts[j] && bin[j] == first_bin;
      if (__all_sync(0xffffffffu, alike)) {
        if (lane == 0) atomicAdd(&sh.bins[first_bin], 128u);
      } else {
#pragma unroll
        for (int j = 0; j < 4; ++j)
          if (counts[j]) atomicAdd(&sh.bins[bin[j]], 1u);
      }
    }
    if (blocks > 1) {
      __syncthreads();
      for (int i = threadIdx.x; i < kPickBins; i += threads)
        if (sh.bins[i] != 0u) add_cluster(joint0 + 4 * i, sh.bins[i]);
    }
    together();
    if (rank == 0) {
      // the bin that holds the left-th largest: the first one from above whose sum with those above it reaches that
      constexpr int each = kPickBins / threads;
      uint32_t own = 0;
      for (int e = 0; e < each; ++e) own += joint[kPickBins - 1 - (threadIdx.x * each + e)];
      uint32_t upto = own;
#pragma unroll
      for (int d = 1; d < 32; d *= 2) {
        const uint32_t y = __shfl_up_sync(0xffffffffu, upto, d);
        if (lane >= d) upto += y;
      }
      if (lane == 31) sh.scan[warp] = upto;
      __syncthreads();
      uint32_t in_front = lane < warp ? sh.scan[lane] : 0u;  // (at most 32 warps)
#pragma unroll
      for (int d = 1; d < 32; d *= 2) in_front += __shfl_xor_sync(0xffffffffu, in_front, d);
      uint32_t above = in_front + upto - own;
      if (above < left && above + own >= left) {
        for (int e = 0; e < each; ++e) {
          const int bin = kPickBins - 1 - (threadIdx.x * each + e);
          const uint32_t here = joint[bin];
          if (above < left && above + here >= left) {
            sh.bin = (uint32_t)bin;
            sh.left = left - above;
            sh.in_bin = here;
          }
          above += here;
        }
      }
    }
    together();
    const uint32_t at_bin = blocks > 1 ? mapa_u32(smem_u32(&sh.bin), 0) : smem_u32(&sh.bin);
    const uint32_t at_left = blocks > 1 ? mapa_u32(smem_u32(&sh.left), 0) : smem_u32(&sh.left);
    prefix |= ld_cluster(at_bin) << shift;
    known |= digits << shift;
    left = ld_cluster(at_left);
    if (blocks > 1) continue;  // (the next pass begins with a barrier before these are written again)
    const bool few = sh.in_bin <= kPickFew;
    if (threadIdx.x == 0) sh.listed = 0u;
    __syncthreads();
    if (!few || pass == 2) continue;
    // Those of the bin are few: each is compared with all of them, which takes the place of the passes that are left (5,205 tokens:
    // most often 150 to 200 are in the first pass's bin).
    uint32_t* list = sh.joint;
    for (int at = begin; at < end; at += kPickStep) {
      const uint4 x4 = numbers_at(at + 4 * lane);
      const uint32_t x[4] = {x4.x, x4.y, x4.z, x4.w};
#pragma unroll
      for (int j = 0; j < 4; ++j)
        if ((x[j] & known) == prefix && x[j] != 0u) list[atomicAdd(&sh.listed, 1u)] = x[j];
    }
    __syncthreads();
    const uint32_t n_listed = sh.listed;
    for (uint32_t i = n_listed + threadIdx.x; i < ((n_listed + 3) & ~3u); i += threads) list[i] = 0u;
    __syncthreads();
    if (threadIdx.x < n_listed) {
      const uint32_t x = list[threadIdx.x];
      uint32_t over = 0, same = 0;
      for (uint32_t i = 0; i < n_listed; i += 4) {
        const uint4 y = *reinterpret_cast<const uint4*>(list + i);
        over += (y.x > x ? 1u : 0u) + (y.y > x ? 1u : 0u) + (y.z > x ? 1u : 0u) + (y.w > x ? 1u : 0u);
        same += (y.x == x ? 1u : 0u) + (y.y == x ? 1u : 0u) + (y.z == x ? 1u : 0u) + (y.w == x ? 1u : 0u);
      }
      if (over < left && over + same >= left) {  // (its equals write the same)
        sh.bin = x;
        sh.left = left - over;
      }
    }
    __syncthreads();
    prefix = sh.bin;
    left = sh.left;
    break;
  }
  // prefix: the least that stays, which is somebody's; left: how many of its equals do, from the front

  // Two counts, of larger ones and of equal ones, side by side in 64 bits.
  auto counts_of = [&](const uint4& x) {
    auto one = [&](uint32_t y) { return (unsigned long long)(y > prefix ? 1u : 0u) << 32 | (y == prefix ? 1u : 0u); };
    return one(x.x) + one(x.y) + one(x.z) + one(x.w);
  };
  unsigned long long own = 0;
  for (int at = begin; at < end; at += kPickStep) own += counts_of(numbers_at(at + 4 * lane));
#pragma unroll
  for (int d = 1; d < 32; d *= 2) own += __shfl_xor_sync(0xffffffffu, own, d);
  if (lane == 0) sh.warp_sums[warp][0] = (uint32_t)(own >> 32), sh.warp_sums[warp][1] = (uint32_t)own;
  __syncthreads();
  if (warp < 2) {
    uint32_t sum = lane < n_warps ? sh.warp_sums[lane][warp] : 0u;
#pragma unroll
    for (int d = 1; d < 32; d *= 2) sum += __shfl_xor_sync(0xffffffffu, sum, d);
    if (lane == 0) sh.counts[warp] = sum;
  }
  together();
  // in front of this warp: the ranks', and the CTA's own warps'
  uint32_t above = 0, equal = 0;
  if (lane < rank) {
    above = ld_cluster(mapa_u32(smem_u32(&sh.counts[0]), lane));
    equal = ld_cluster(mapa_u32(smem_u32(&sh.counts[1]), lane));
  }
  if (lane < warp) above += sh.warp_sums[lane][0], equal += sh.warp_sums[lane][1];
#pragma unroll
  for (int d = 1; d < 32; d *= 2) {
    above += __shfl_xor_sync(0xffffffffu, above, d);
    equal += __shfl_xor_sync(0xffffffffu, equal, d);
  }
  for (int at = begin; at < end; at += kPickStep) {
    const int token = at + 4 * lane;
    const uint4 x4 = numbers_at(token);
    const unsigned long long here = counts_of(x4);
    unsigned long long upto = here;
#pragma unroll
    for (int d = 1; d < 32; d *= 2) {
      const unsigned long long y = __shfl_up_sync(0xffffffffu, upto, d);
      if (lane >= d) upto += y;
    }
    const unsigned long long step = __shfl_sync(0xffffffffu, upto, 31);
    uint32_t over = above + (uint32_t)((upto - here) >> 32), same = equal + (uint32_t)(upto - here);
    const uint32_t x[4] = {x4.x, x4.y, x4.z, x4.w};
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      if (x[j] > prefix || (x[j] == prefix && same < left)) put(first + (int)(over + min(same, left)), token + j);
      over += x[j] > prefix ? 1u : 0u;
      same += x[j] == prefix ? 1u : 0u;
    }
    above += (uint32_t)(step >> 32);
    equal += (uint32_t)step;
  }
  together();  // nobody's shared memory goes while others read it
}

constexpr int kMoveThreads = 256;

// Places of the pages that are filled, one after another: (page of the list, head, token in the page).
template <int kHd, int kKind, int kUnits>
__global__ void __launch_bounds__(kMoveThreads)
kv_move_kernel(KvPool pool, KvArrays from, KvArrays into, const int* __restrict__ kept, long long units) {
  constexpr int kRowBytes = KvRow<kHd, kKind>::kBytes, kExps = KvRow<kHd, kKind>::kExps, kLanes = kRowBytes / 16, kGroups = kMoveThreads / kLanes;
  const int part = threadIdx.x % kLanes;
  const long long unit0 = (long long)blockIdx.x * (kGroups * kUnits) + threadIdx.x / kLanes;
  size_t to[kUnits], at[kUnits];
  long long number[kUnits];  // in the list of kept tokens
  int head[kUnits], page0[kUnits];
  bool live[kUnits];
#pragma unroll
  for (int i = 0; i < kUnits; ++i) {  // (a batch's arrays were there before whatever kernel is still running)
    const long long unit = unit0 + i * kGroups;
    live[i] = unit < units;
    if (!live[i]) continue;
    const int offset = (int)(unit & (pool.page_size - 1));
    const long long in_pages = unit >> pool.page_shift;
    const int entry = (int)(in_pages / pool.kv_heads);
    head[i] = (int)(in_pages % pool.kv_heads);
    int lo = 0, hi = into.n_seq - 1;
    while (lo < hi) {  // the last sequence that begins at or before the page; ones without pages share their successor's start
      const int mid = (lo + hi + 1) >> 1;
      if (into.seqs[mid].page0 <= entry) lo = mid;
      else hi = mid - 1;
    }
    const KvSeq dst = into.seqs[lo];
    const int slot = ((entry - dst.page0) << pool.page_shift) + offset;
    live[i] = slot < dst.len;
    number[i] = (long long)(dst.row0 + slot) * pool.kv_heads + head[i];
    page0[i] = from.seqs[lo].page0;
    to[i] = (((size_t)into.pages[entry] * pool.kv_heads + head[i]) << pool.page_shift) + offset;
  }
  wait_for_previous_kernel();
  int token[kUnits];
#pragma unroll
  for (int i = 0; i < kUnits; ++i)
    if (live[i]) token[i] = kept[number[i]];
#pragma unroll
  for (int i = 0; i < kUnits; ++i) {
    if (!live[i]) continue;
    const size_t page = (size_t)from.pages[page0[i] + (token[i] >> pool.page_shift)];
    at[i] = ((page * pool.kv_heads + head[i]) << pool.page_shift) + (token[i] & (pool.page_size - 1));
  }
  uint4 xk[kUnits], xv[kUnits];
  uint32_t ek[kUnits], ev[kUnits];
  float w[kUnits];
#pragma unroll
  for (int i = 0; i < kUnits; ++i) {
    if (!live[i]) continue;
    xk[i] = ldg16(pool.k + at[i] * kRowBytes + part * 16);
    xv[i] = ldg16(pool.v + at[i] * kRowBytes + part * 16);
    if (kExps > 0 && part < kExps) {  // (a row of E2M1 codes has as many lanes as exponents)
      ek[i] = pool.k_exp[at[i] * kExps + part];
      ev[i] = pool.v_exp[at[i] * kExps + part];
    }
    if (part == 0) w[i] = pool.weights[at[i]];
  }
#pragma unroll
  for (int i = 0; i < kUnits; ++i) {
    if (!live[i]) continue;
    stg16(pool.k + to[i] * kRowBytes + part * 16, xk[i]);
    stg16(pool.v + to[i] * kRowBytes + part * 16, xv[i]);
    if (kExps > 0 && part < kExps) {
      pool.k_exp[to[i] * kExps + part] = (uint8_t)ek[i];
      pool.v_exp[to[i] * kExps + part] = (uint8_t)ev[i];
    }
    if (part == 0) pool.weights[to[i]] = w[i];
  }
}

template <int kHd, int kKind>
cudaError_t move(const litevggt_kv_cache& c, const litevggt_kv_batch& from, const litevggt_kv_batch& into, const int* kept, long long pages, cudaStream_t s) {
  constexpr int kLanes = KvRow<kHd, kKind>::kBytes / 16, kGroups = kMoveThreads / kLanes;
  static_assert(KvRow<kHd, kKind>::kExps <= kLanes, "");
  const long long units = pages * c.cfg.kv_heads * c.cfg.page_size, blocks = (units + kGroups - 1) / kGroups;
  if (blocks <= (long long)c.num_sms * (2048 / kMoveThreads))
    return launch(kv_move_kernel<kHd, kKind, 1>, dim3((unsigned)blocks), kMoveThreads, 0, s, c.pool, kv_arrays(from), kv_arrays(into), kept, units);
  return launch(kv_move_kernel<kHd, kKind, 2>, dim3((unsigned)((blocks + 1) / 2)), kMoveThreads, 0, s, c.pool, kv_arrays(from), kv_arrays(into), kept, units);
}

// Blocks of a cluster at most: 16 SMs where the device has that many together (more than the eight that every one has to offer).
// Looked up once for each device.
int pick_blocks() {
  static std::atomic<unsigned long long> asked{0}, fits{0};
  int device = 0;
  if (cudaGetDevice(&device) != cudaSuccess) return kPickPortableBlocks;
  const unsigned long long bit = 1ull << (device & 63);
  if ((asked.load(std::memory_order_acquire) & bit) == 0) {
    const void* kernel = reinterpret_cast<const void*>(kv_pick_kernel<kPickMostThreads>);
    cudaLaunchAttribute attr;
    attr.id = cudaLaunchAttributeClusterDimension;
    attr.val.clusterDim.x = kPickMostBlocks;
    attr.val.clusterDim.y = attr.val.clusterDim.z = 1;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3(kPickMostBlocks);
    cfg.blockDim = dim3(kPickMostThreads);
    cfg.dynamicSmemBytes = kPickMostHeld * 4;
    cfg.attrs = &attr;
    cfg.numAttrs = 1;
    int clusters = 0;
    bool set = true;
    for (const void* k : {kernel, reinterpret_cast<const void*>(kv_pick_kernel<kPickThreads>)})
      set = set && cudaFuncSetAttribute(k, cudaFuncAttributeMaxDynamicSharedMemorySize, kPickMostHeld * 4) == cudaSuccess &&
            cudaFuncSetAttribute(k, cudaFuncAttributeNonPortableClusterSizeAllowed, 1) == cudaSuccess;
    if (set && cudaOccupancyMaxActiveClusters(&clusters, kernel, &cfg) == cudaSuccess && clusters > 0)
      fits.fetch_or(bit);
    else (void)cudaGetLastError();
    asked.fetch_or(bit, std::memory_order_release);
  }
  return (fits.load(std::memory_order_relaxed) & bit) != 0 ? kPickMostBlocks : kPickPortableBlocks;
}

}  // namespace

cudaError_t launch_kv_evict(const litevggt_kv_cache& c, const litevggt_kv_batch& from, const litevggt_kv_batch& into, int first, int last,
                            int* kept, cudaStream_t s, int* launches) {
  const long long pairs = (long long)from.seqs.size() * c.cfg.kv_heads;
  // CTAs of a head: as many as there is room for, where its tokens are more than eight for each of a CTA's threads; and twice the threads
  // where that is not enough.
  int longest = 0, blocks = 1;
  for (const KvSeq& q : from.seqs) longest = std::max(longest, q.len);
  const int most = pick_blocks();
  while (blocks < most && 2 * blocks * pairs <= 2ll * c.num_sms && longest > blocks * 8 * kPickThreads) blocks *= 2;
  const int threads = longest > blocks * 16 * kPickThreads && blocks * pairs <= 2ll * c.num_sms ? kPickMostThreads : kPickThreads;
  const int warps = threads / 32;
  const long long run = round_up(((long long)longest + 3 + blocks * warps - 1) / (blocks * warps), kPickStep);
  const int held = (int)std::min(run, (long long)kPickMostHeld / warps);
  auto kernel = threads == kPickMostThreads ? kv_pick_kernel<kPickMostThreads> : kv_pick_kernel<kPickThreads>;
  cudaError_t e = launch_clusters(blocks, true, kernel, dim3((unsigned)(pairs * blocks)), (unsigned)threads, (size_t)held * warps * 4, s, c.pool,
                                  kv_arrays(from), kv_arrays(into), first, last, blocks, held, kept);
  ++*launches;
  const long long pages = kv_page_count(into, c.cfg.page_size);
  if (e != cudaSuccess || pages == 0) return e;
  ++*launches;
  const bool wide = c.cfg.head_dim == 128;
  if (c.cfg.dtype == LITEVGGT_KV_E2M1) return wide ? move<128, LITEVGGT_KV_E2M1>(c, from, into, kept, pages, s) : move<64, LITEVGGT_KV_E2M1>(c, from, into, kept, pages, s);
  if (c.cfg.dtype == LITEVGGT_KV_E4M3) return wide ? move<128, LITEVGGT_KV_E4M3>(c, from, into, kept, pages, s) : move<64, LITEVGGT_KV_E4M3>(c, from, into, kept, pages, s);
  return wide ? move<128, LITEVGGT_KV_BF16>(c, from, into, kept, pages, s) : move<64, LITEVGGT_KV_BF16>(c, from, into, kept, pages, s);
}

}  // namespace lv
