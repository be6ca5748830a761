// Paged cache in 8 bits, eviction: of every (sequence, layer, KV head) that is longer than the budget the first and last tokens
// and the heaviest of the others are kept, and move together where they stand. A cluster of CTAs takes a head of a layer.
//
// Choice: each CTA has a share of the tokens. A radix select over the weights as ordered integers, 8 bits a pass: histograms in shared
// memory, read by every CTA of the cluster; a CTA also adds up what the shares before its own keep, so that the kept tokens can be
// listed in order without another exchange. It ends when there is room for all weights with the digits so far.
// Move: the cluster goes over the new places 128 a CTA at a time; every CTA reads the tokens that come to its places, a cluster barrier,
// then they are written. A token never moves up, so what a later round reads lies behind everything that an earlier round
// writes, and the reads of the next two rounds are under way while one writes.
//
// Bound by latency: a cluster barrier and the memory's latency a round, few bytes in flight beside what the memory takes. 131072 tokens of 8
// heads cut to 65536: 100 us (277 MB, 0.41 of a copy); 4 layers of 8 sequences of 9000 to 32000 tokens to 12288: 264 us (0.81); four
// sequences of 900 to 1500 tokens to 1024: 21 us, of which the passes of the select and one round each are latency alone. A head is a chain of rounds, and there are only as many
// heads as the cache has: clusters are the largest, up to 16, with no more than four times as many CTAs as the device holds (at 131072 tokens
// clusters of 16 104 us, of 8 133, of 4 193; the 256 heads of 4 layers and 8 sequences 265 us with four times as many, in clusters of 4; with
// one, two and eight times 369, 283 and 303).
// On the way, at 131072 tokens: histograms of other CTAs read one after another 11000 cycles a pass, now by all lanes at once;
// cluster barriers with release and acquire of everything 117 us, with only the shared memory's order needed 103; mbarriers in their place
// 107; larger rounds, choice and move in two kernels, and warps that follow each other's progress by counters were not faster (103, 278
// and 132 to 178).
#include <math.h>

#include <atomic>

#include <cooperative_groups.h>

#include "common.cuh"
#include "paged.h"
#include "paged8.h"

namespace cg = cooperative_groups;

namespace vr {

namespace {

constexpr int kThreads = 512, kWarps = kThreads / 32, kCtas = 2, kMostCluster = 16;
constexpr int kBins = 256;
constexpr int kTile = 128;                               // new places of a CTA in a round
constexpr int kPieces = kTile * 2 * 8 / kThreads;        // 16-byte pieces of a thread in a round
constexpr int kStages = 3, kPlaces = kStages + 1;        // rounds on their way; and found
constexpr int kMostCached = kStages * kTile * 2 * kHeadDim / 4;   // weights of a CTA's share that shared memory holds

struct Evict {
  Paged p;
  unsigned char *codes, *scale;                          // of the first layer
  float* mass;
  int32_t *kept, *new_len, *gone, *dev_status;
  int n_layers, budget, n_first, n_last;
};

struct Shared {
  union {
    uint4 piece[kStages][kPieces][kThreads];             // the move: a thread's own
    uint32_t cached[kMostCached];                        // the choice: weights of the CTA's share
  };
  int hist[2][kBins];
  int wsum[kWarps][2];
  // of a pass: the digit, how many of the others are above it, of those how many in the shares before this CTA's, how many with it in
  // those shares, and whether there is room for all that have it
  int bin, above, above_before, equal_before, all;
  int bad;                                               // a page of this CTA's share is out of range
  int from[kPlaces][kTile], to[kPlaces][kTile];          // rows of the codes, K, of a place's token and of the place; -1: none
  float weight[kPlaces][kTile];
  unsigned char shift[kPlaces][2][kTile];                // its codes go down by 2^shift
  unsigned char byte[kPlaces][2][kTile];                 // its new block's scale
};

// Weights in an order of unsigned integers: NaN above everything, -0 as 0.
__device__ __forceinline__ uint32_t order(float x) {
  const uint32_t b = __float_as_uint(x);
  if (x != x) return 0xffffffffu;
  if (x == 0.f) return 0x80000000u;
  return b >> 31 ? ~b : b | 0x80000000u;
}

__global__ void __launch_bounds__(kThreads, kCtas) paged8_evict_kernel(Evict a) {
  extern __shared__ __align__(16) unsigned char smem[];
  Shared& c = *reinterpret_cast<Shared*>(smem);
  cg::cluster_group cluster = cg::this_cluster();
  const int ctas = (int)cluster.num_blocks();
  const Paged& p = a.p;
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, rank = (int)cluster.block_rank();
  const unsigned head = blockIdx.x / ctas, G = p.G;
  const int g = (int)(head % G), layer = (int)(head / G % a.n_layers), s = (int)(head / G / a.n_layers);
  const int in_page = (1 << p.page_log2) - 1;
  pdl_trigger();
  if (tid < kBins) c.hist[0][tid] = 0;
  if (tid == 0) c.bad = 0;
  __syncthreads();
  pdl_wait();
  const int len = __ldg(p.kv_len + s);
  const int32_t* table = p.table + (int64_t)s * p.max_pages;
  int32_t* kept = a.kept + (int64_t)head * a.budget;
  unsigned char* codes = a.codes + (int64_t)layer * p.layer_rows * kHeadDim;
  unsigned char* scale = a.scale + (int64_t)layer * (p.layer_rows >> kBlockLog2);
  float* mass = a.mass + (int64_t)layer * (p.layer_rows / 2);
  const bool wrong = len < 0 || len > kMaxLen || len > ((int64_t)p.max_pages << p.page_log2);
  auto close = [&](int keep, bool bad) {                 // by one thread of the sequence
    if (bad) raise_status(a.dev_status, VARRATE_ERR_CORRUPT);
    a.new_len[s] = keep;
    if (a.gone && !bad) a.gone[s] += len - keep;
  };
  const bool first = rank == 0 && tid == 0 && g == 0 && layer == 0;
  if (wrong || len <= a.budget) {                        // (the same for the cluster; nothing of the pages is looked at)
    const int keep = wrong ? 0 : len;
    for (int64_t i = (int64_t)rank * kThreads + tid; i < a.budget; i += ctas * kThreads) kept[i] = i < keep ? (int)i : -1;
    if (first) close(keep, wrong);
    return;
  }
  // this CTA's share of the tokens; mid0 .. mid1 - 1 are those that are chosen from, more than there is room for
  const int share = (int)(((int64_t)len + ctas * 32 - 1) / (ctas * 32)) * 32;
  const int lo = (int)min((int64_t)rank * share, (int64_t)len), hi = (int)min((int64_t)lo + share, (int64_t)len);
  const int mid0 = a.n_first, mid1 = len - a.n_last, b0 = max(lo, mid0), b1 = min(hi, mid1);
  int room = a.budget - a.n_first - a.n_last;            // for the others, and then for those with the last digit chosen
  const bool some = room > 0;
  auto weight_at = [&](int i) {
    const int page = __ldg(table + (i >> p.page_log2));
    if ((unsigned)page >= (unsigned)p.n_pages) { c.bad = 1; return 0u; }
    return order(mass[mass_at(p, page, g, i & in_page)]);
  };
  const bool in_cache = share <= kMostCached;
#pragma unroll 8
  for (int i = lo + tid; i < hi; i += kThreads) {
    const uint32_t k = weight_at(i);
    if (in_cache) c.cached[i - lo] = k;
    if (i >= b0 && i < b1) atomicAdd(&c.hist[0][k >> 24], 1);
  }
  auto key_at = [&](int i) { return in_cache ? c.cached[i - lo] : weight_at(i); };
  uint32_t least = 0;                                    // the digits of the least weight kept so far, and where the last of them is
  int low = 24, sure_before = 0, equal_before = 0;
  bool bad = false;
  for (int pass = 0;; ++pass, low -= 8) {
    int* hist = c.hist[pass & 1];
    if (pass > 0)
      for (int i = b0 + tid; i < b1; i += kThreads) {
        const uint32_t k = key_at(i);
        if ((k ^ least) >> (low + 8) == 0) atomicAdd(&hist[k >> low & (kBins - 1)], 1);
      }
    cluster.sync();
    if (pass == 0) {
      bad = __any_sync(0xffffffffu, lane < ctas && *cluster.map_shared_rank(&c.bad, min(lane, ctas - 1)) != 0);
      if (bad || !some) break;                           // (the same for the cluster)
    }
    if (tid < kBins) c.hist[~pass & 1][tid] = 0;         // (read by every CTA before it came to this barrier)
    // a digit a thread, the highest one first; how many are above it
    int n = 0, mine = 0;
    if (tid < kBins) {
#pragma unroll
      for (int i = 0; i < kMostCluster; ++i) {
        const int x = i < ctas ? cluster.map_shared_rank(hist, i)[kBins - 1 - tid] : 0;
        n += x;
        if (i < rank) mine += x;
      }
    }
    int incl = n, incl_mine = mine;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const int y = __shfl_up_sync(0xffffffffu, incl, o), z = __shfl_up_sync(0xffffffffu, incl_mine, o);
      if (lane >= o) { incl += y; incl_mine += z; }
    }
    if (lane == 31) { c.wsum[warp][0] = incl; c.wsum[warp][1] = incl_mine; }
    __syncthreads();
    if (tid < kBins) {
      int above = incl - n, above_mine = incl_mine - mine;
      for (int i = 0; i < warp; ++i) { above += c.wsum[i][0]; above_mine += c.wsum[i][1]; }
      if (above < room && above + n >= room) {
        c.bin = kBins - 1 - tid;
        c.above = above;
        c.above_before = above_mine;
        c.equal_before = mine;
        c.all = above + n == room;
      }
    }
    __syncthreads();
    least |= (uint32_t)c.bin << low;
    room -= c.above;
    sure_before += c.above_before;
    equal_before = c.equal_before;
    if (c.all || low == 0) break;
  }
  if (bad) {
    for (int64_t i = (int64_t)rank * kThreads + tid; i < a.budget; i += ctas * kThreads) kept[i] = -1;
    if (first) close(0, true);
    cluster.sync();                                      // no CTA leaves while its shared memory may be read
    return;
  }
  {
    // A warp's tokens of the share: those kept for sure (the first, the last, the heavier), those with the least digits.
    const int per = (hi - lo + kWarps * 32 - 1) / (kWarps * 32) * 32;
    const int w0 = min(hi, lo + warp * per), w1 = min(hi, w0 + per);
    auto kind = [&](int i, bool& sure, bool& equal) {
      const bool mid = i >= mid0 && i < mid1;
      const uint32_t k = i < w1 && mid && some ? key_at(i) >> low : 0u;
      sure = i < w1 && (!mid || (some && k > least >> low));
      equal = i < w1 && mid && some && k == least >> low;
    };
    int gt = 0, eq = 0;
    for (int i = w0; i < w1; i += 32) {
      bool sure, equal;
      kind(i + lane, sure, equal);
      gt += __popc(__ballot_sync(0xffffffffu, sure));
      eq += __popc(__ballot_sync(0xffffffffu, equal));
    }
    __syncthreads();                                     // (wsum of the last pass)
    if (lane == 0) { c.wsum[warp][0] = gt; c.wsum[warp][1] = eq; }
    __syncthreads();
    int x = lane < warp ? c.wsum[lane][0] : 0, y = lane < warp ? c.wsum[lane][1] : 0;
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) {
      x += __shfl_xor_sync(0xffffffffu, x, o);
      y += __shfl_xor_sync(0xffffffffu, y, o);
    }
    sure_before += x + min(lo, mid0) + max(0, lo - mid1);
    equal_before += y;
    for (int i = w0; i < w1; i += 32) {
      bool sure, equal;
      kind(i + lane, sure, equal);
      const unsigned below = (1u << lane) - 1, ms = __ballot_sync(0xffffffffu, sure), me = __ballot_sync(0xffffffffu, equal);
      const int e = equal_before + __popc(me & below);
      if (sure || (equal && e < room)) kept[sure_before + __popc(ms & below) + min(e, room)] = i + lane;
      sure_before += __popc(ms);
      equal_before += __popc(me);
    }
    if (first) close(a.budget, false);
  }
  cluster.sync();                                        // the list is complete

  // The move. A place's token is found in steps, a round apart, so that no load is waited for: which one (a), its page and that of the
  // place (b), scale and weight (c). Threads 0 .. 127 take the keys of the CTA's places, 128 .. 255 the values.
  const int keep = a.budget, round_places = ctas * kTile, to_v = (int)G << p.page_log2;
  const int rounds = (int)(((int64_t)keep + round_places - 1) / round_places);
  int round = 0;
  while ((int64_t)(round + 1) * round_places <= keep && __ldcg(kept + (int64_t)(round + 1) * round_places - 1) == (round + 1) * round_places - 1)
    ++round;                                             // these stay
  const int kv = tid / kTile & 1, place = tid % kTile;
  const bool finds = tid < 2 * kTile;
  auto at_place = [&](int r) { return (int64_t)r * round_places + rank * kTile + place; };
  int src_a = -1, src_b = -1, page_b = 0, dst_b = 0;
  auto find_a = [&](int r) { src_a = finds && r < rounds && at_place(r) < keep ? __ldcg(kept + at_place(r)) : -1; };
  auto find_b = [&](int r) {
    src_b = src_a;
    if (src_b < 0) return;
    page_b = __ldg(table + (src_b >> p.page_log2));
    dst_b = __ldg(table + (at_place(r) >> p.page_log2));
  };
  int byte_c = 0, from_c = -1, to_c = -1;
  float weight_c = 0.f;
  auto find_c = [&](int r) {
    byte_c = 0;
    from_c = to_c = -1;
    if (src_b < 0) return;
    from_c = (int)page_row(p, page_b, 0, g, src_b & in_page);
    to_c = (int)page_row(p, dst_b, 0, g, (int)(at_place(r) & in_page));
    byte_c = scale[scale_at(from_c + (kv ? to_v : 0))];
    if (kv == 0) weight_c = mass[mass_at(p, page_b, g, src_b & in_page)];
  };
  auto found = [&](int at) {
    if (!finds) return;
    int most = byte_c;
#pragma unroll
    for (int o = 1; o < kBlock; o <<= 1) most = max(most, __shfl_xor_sync(0xffffffffu, most, o));
    c.shift[at][kv][place] = (unsigned char)(most - byte_c);
    c.byte[at][kv][place] = (unsigned char)most;
    if (kv == 0) {
      c.from[at][place] = from_c;
      c.to[at][place] = to_c;
      c.weight[at][place] = weight_c;
    }
  };
  const int token0 = tid >> 4, kv_p = tid >> 3 & 1, off = 16 * (tid & 7);   // of this thread's first piece; the others are kThreads / 16 tokens on
  auto load = [&](int r) {
#pragma unroll
    for (int i = 0; i < kPieces; ++i) {
      const int from = c.from[r % kPlaces][token0 + i * (kThreads / 16)];
      if (from >= 0) cp_async16(smem_addr(&c.piece[r % kStages][i][tid]), codes + (int64_t)(from + (kv_p ? to_v : 0)) * kHeadDim + off, 16);
    }
    cp_async_commit();
  };
  // Before the first round: the places of the next kStages rounds, and the loads of all of them but one.
  {
    int src[kStages], page[kStages], dst[kStages];
#pragma unroll
    for (int i = 0; i < kStages; ++i) { find_a(round + i); src[i] = src_a; }
    find_a(round + kStages);
    const int next = src_a;
#pragma unroll
    for (int i = 0; i < kStages; ++i) {
      src_a = src[i];
      find_b(round + i);
      page[i] = page_b; dst[i] = dst_b;
    }
    int byte[kStages], from[kStages], to[kStages];
    float weight[kStages];
#pragma unroll
    for (int i = 0; i < kStages; ++i) {
      src_b = src[i]; page_b = page[i]; dst_b = dst[i];
      find_c(round + i);
      byte[i] = byte_c; from[i] = from_c; to[i] = to_c; weight[i] = weight_c;
    }
    src_a = next;
    find_b(round + kStages);
    find_a(round + kStages + 1);
#pragma unroll
    for (int i = 0; i < kStages; ++i) {
      byte_c = byte[i]; from_c = from[i]; to_c = to[i]; weight_c = weight[i];
      found((round + i) % kPlaces);
    }
  }
  __syncthreads();
  for (int r = round; r < round + kStages - 1; ++r) load(r);
  find_c(round + kStages);
  find_b(round + kStages + 1);
  find_a(round + kStages + 2);
  for (; round < rounds; ++round) {
    cp_async_wait<kStages - 2>();                        // this thread's pieces of the round
    // Every CTA has read this round's tokens before one writes. Nothing that a round writes is read later, so the barrier releases
    // nothing, which would wait for the stores before it.
    asm volatile("barrier.cluster.arrive.relaxed.aligned;\n" ::: "memory");
    load(round + kStages - 1);
    found((round + kStages) % kPlaces);
    find_c(round + kStages + 1);
    find_b(round + kStages + 2);
    find_a(round + kStages + 3);
    asm volatile("barrier.cluster.wait.aligned;\n" ::: "memory");
    const int at = round % kPlaces;
#pragma unroll
    for (int i = 0; i < kPieces; ++i) {
      const int token = token0 + i * (kThreads / 16), to = c.to[at][token], shift = c.shift[at][kv_p][token];
      if (to < 0) continue;
      uint4 y = c.piece[round % kStages][i][tid];
      if (shift) {
        const Rescale by(shift);
        y = make_uint4(by.four(y.x), by.four(y.y), by.four(y.z), by.four(y.w));
      }
      *reinterpret_cast<uint4*>(codes + (int64_t)(to + (kv_p ? to_v : 0)) * kHeadDim + off) = y;
    }
    if (finds) {
      const int to = c.to[at][place];
      if (to >= 0) {
        if ((place & (kBlock - 1)) == 0) scale[scale_at(to + (kv ? to_v : 0))] = c.byte[at][kv][place];
        if (kv == 0) mass[mass_at(p, (to >> p.page_log2) / (2 * (int)G), g, to & in_page)] = c.weight[at][place];
      }
    }
    __syncthreads();                                     // the places found; this round's are written again
  }
  cp_async_wait<0>();
  cluster.sync();
}

}  // namespace

int launch_paged8_evict(const Paged8& c, int layer, int n_layers, int budget, int n_first, int n_last, int32_t* kept,
                        int32_t* new_len, int32_t* gone, int32_t* dev_status, int num_sms, cudaStream_t st) {
  const Paged& p = c.p;
  Evict a;
  a.p = p;
  a.codes = p.pool + (int64_t)layer * p.layer_rows * kHeadDim;
  a.scale = c.scale + (int64_t)layer * (p.layer_rows >> kBlockLog2);
  a.mass = c.mass + (int64_t)layer * (p.layer_rows / 2);
  a.kept = kept; a.new_len = new_len; a.gone = gone; a.dev_status = dev_status;
  a.n_layers = n_layers; a.budget = budget; a.n_first = n_first; a.n_last = n_last;
  static std::atomic<int> smem_set[64];
  int dev = 0;
  if (cudaGetDevice(&dev) != cudaSuccess || dev < 0 || dev >= 64 || smem_set[dev].load(std::memory_order_acquire) == 0) {
    if (cudaFuncSetAttribute(paged8_evict_kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)sizeof(Shared)) != cudaSuccess ||
        cudaFuncSetAttribute(paged8_evict_kernel, cudaFuncAttributeNonPortableClusterSizeAllowed, 1) != cudaSuccess)
      return -1;
    if (dev >= 0 && dev < 64) smem_set[dev].store(1, std::memory_order_release);
  }
  // CTAs of a cluster, a power of two: up to four times what the device holds at once, but none without a tile of the longest list
  const int64_t heads = (int64_t)p.S * n_layers * p.G, longest = (int64_t)p.max_pages << p.page_log2, list = budget < longest ? budget : longest;
  int ctas = 1;
  while (ctas < kMostCluster && 2 * ctas * heads <= 4 * kCtas * num_sms && (int64_t)ctas * kTile < list) ctas *= 2;
  cudaLaunchAttribute attr[2];
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  attr[1].id = cudaLaunchAttributeClusterDimension;
  attr[1].val.clusterDim.x = (unsigned)ctas; attr[1].val.clusterDim.y = 1; attr[1].val.clusterDim.z = 1;
  cudaLaunchConfig_t lc = {};
  lc.gridDim = dim3((unsigned)(heads * ctas));
  lc.blockDim = dim3(kThreads);
  lc.dynamicSmemBytes = sizeof(Shared);
  lc.stream = st;
  lc.attrs = attr;
  lc.numAttrs = 2;
  return cudaLaunchKernelEx(&lc, paged8_evict_kernel, a) == cudaSuccess ? 1 : -1;
}

}  // namespace vr
