// Paged cache in 8 bits, eviction: of every (sequence, layer, KV head) that is longer than the budget the first and last tokens
// and the heaviest of the others are kept, and move together where they stand.
//
// A cluster of eight CTAs takes a head of a layer. Which are kept: a radix select over the weights as ordered integers (11, 11
// and 10 bits; histograms in shared memory, summed over the cluster), the kept tokens listed in order into `kept`. Move: the cluster
// goes over the new places 1024 at a time; every CTA reads the 128 tokens that come to its places, a cluster barrier, then they are
// written. A token never moves up, so what a later round reads lies behind everything that an earlier round writes, and the reads of the
// next round are under way while a round writes.
#include <math.h>

#include <atomic>

#include <cooperative_groups.h>

#include "common.cuh"
#include "paged.h"
#include "paged8.h"

namespace cg = cooperative_groups;

namespace vr {

namespace {

constexpr int kThreads = 512, kWarps = kThreads / 32, kCluster = 8;
constexpr int kBins = 2048;
constexpr int kTile = 128;                               // new places of a CTA in a round
constexpr int kPieces = kTile * 2 * 8 / kThreads;        // 16-byte pieces of a thread in a round
constexpr int kMostCached = 40960;                       // weights of a CTA's share that shared memory holds

struct Evict {
  Paged p;
  unsigned char *codes, *scale;                          // of the first layer
  float* mass;
  int32_t *kept, *new_len, *gone, *dev_status;
  int n_layers, budget, n_first, n_last, cache;
};

struct Shared {
  int hist[kBins];
  int wsum[kWarps][2];
  int bin, above;                                        // of a pass: the digit, and how many are above it
  int gt, eq, bad;                                       // of this CTA's share
  int64_t from[2][kTile];                                // row of the codes that a place's token comes from, -1: none
  int64_t to[kTile];
  unsigned char shift[2][2][kTile];                      // its codes go down by 2^shift
  unsigned char byte[2][2][kTile];                       // its new block's scale
};

// Weights in an order of unsigned integers: NaN above everything, -0 as 0.
__device__ __forceinline__ uint32_t order(float x) {
  const uint32_t b = __float_as_uint(x);
  if (x != x) return 0xffffffffu;
  if (x == 0.f) return 0x80000000u;
  return b >> 31 ? ~b : b | 0x80000000u;
}

__global__ void __cluster_dims__(kCluster, 1, 1) __launch_bounds__(kThreads, 1) paged8_evict_kernel(Evict a) {
  extern __shared__ __align__(16) unsigned char smem[];
  Shared& c = *reinterpret_cast<Shared*>(smem);
  uint32_t* cached = reinterpret_cast<uint32_t*>(smem + sizeof(Shared));
  cg::cluster_group cluster = cg::this_cluster();
  const Paged& p = a.p;
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, rank = (int)cluster.block_rank();
  const unsigned head = blockIdx.x / kCluster, G = p.G;
  const int g = (int)(head % G), layer = (int)(head / G % a.n_layers), s = (int)(head / G / a.n_layers);
  const int in_page = (1 << p.page_log2) - 1;
  pdl_trigger();
  pdl_wait();
  const int len = __ldg(p.kv_len + s);
  const int32_t* table = p.table + (int64_t)s * p.max_pages;
  int32_t* kept = a.kept + (int64_t)head * a.budget;
  unsigned char* codes = a.codes + (int64_t)layer * p.layer_rows * kHeadDim;
  unsigned char* scale = a.scale + (int64_t)layer * (p.layer_rows >> kBlockLog2);
  float* mass = a.mass + (int64_t)layer * (p.layer_rows / 2);
  bool bad = len < 0 || len > kMaxLen || len > ((int64_t)p.max_pages << p.page_log2);

  // this CTA's share of the tokens, and of the pages
  const int share = bad ? 0 : (int)(((int64_t)len + kCluster * 32 - 1) / (kCluster * 32)) * 32;
  const int lo = (int)min((int64_t)rank * share, (int64_t)max(len, 0)), hi = (int)min((int64_t)lo + share, (int64_t)max(len, 0));
  if (tid == 0) c.bad = 0;
  __syncthreads();
  if (!bad) {
    bool wrong = false;
    const int pages = (len >> p.page_log2) + ((len & in_page) != 0);
    for (int i = rank * kThreads + tid; i < pages; i += kCluster * kThreads) wrong |= (unsigned)__ldg(table + i) >= (unsigned)p.n_pages;
    if (wrong) c.bad = 1;
  }
  cluster.sync();                                        // (every CTA of the cluster runs)
  for (int i = 0; i < kCluster; ++i) bad |= *cluster.map_shared_rank(&c.bad, i) != 0;
  const int keep = bad ? 0 : min(len, a.budget);
  if (rank == 0 && tid == 0) {
    if (bad) raise_status(a.dev_status, VARRATE_ERR_CORRUPT);
    if (g == 0 && layer == 0) {
      a.new_len[s] = keep;
      if (a.gone && !bad) a.gone[s] += len - keep;
    }
  }
  for (int64_t i = keep + (int64_t)rank * kThreads + tid; i < a.budget; i += kCluster * kThreads) kept[i] = -1;
  if (bad || len <= a.budget) {                          // (the same for the cluster)
    for (int i = rank * kThreads + tid; i < keep; i += kCluster * kThreads) kept[i] = i;
    cluster.sync();                                      // no CTA leaves while its shared memory may be read
    return;
  }

  // ---------------------------------------------------------------- which are kept
  const int mid0 = a.n_first, mid1 = len - a.n_last;     // the others; more than there is room for
  auto weight_at = [&](int i) {
    return order(mass[mass_at(p, __ldg(table + (i >> p.page_log2)), g, i & in_page)]);
  };
  const bool in_cache = share <= a.cache;
  if (in_cache)
    for (int i = lo + tid; i < hi; i += kThreads) cached[i - lo] = weight_at(i);
  auto key_at = [&](int i) { return in_cache ? cached[i - lo] : weight_at(i); };
  const int b0 = max(lo, mid0), b1 = min(hi, mid1);
  int room = a.budget - a.n_first - a.n_last;            // for the others, and then for those equal to the least kept
  uint32_t least = 0;                                    // its digits so far
  for (int pass = 0; pass < 3 && room > 0; ++pass) {     // (room stays above 0 once it is)
    const int shift = pass == 0 ? 21 : pass == 1 ? 10 : 0, bins = pass == 2 ? 1024 : 2048;
    for (int i = tid; i < kBins; i += kThreads) c.hist[i] = 0;
    __syncthreads();
    for (int i = b0 + tid; i < b1; i += kThreads) {
      const uint32_t k = key_at(i);
      if (pass == 0 || (k ^ least) >> (shift + (pass == 2 ? 10 : 11)) == 0) atomicAdd(&c.hist[k >> shift & (bins - 1)], 1);
    }
    cluster.sync();
    // four digits a thread, the highest ones first; how many are above each
    int n[4], sum = 0;
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const int bin = kBins - 1 - 4 * tid - j;
      n[j] = 0;
      for (int i = 0; i < kCluster; ++i) n[j] += cluster.map_shared_rank(c.hist, i)[bin];
      sum += n[j];
    }
    int incl = sum;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const int y = __shfl_up_sync(0xffffffffu, incl, o);
      if (lane >= o) incl += y;
    }
    if (lane == 31) c.wsum[warp][0] = incl;
    __syncthreads();
    int above = incl - sum;
    for (int i = 0; i < warp; ++i) above += c.wsum[i][0];
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      if (above < room && above + n[j] >= room) { c.bin = kBins - 1 - 4 * tid - j; c.above = above; }
      above += n[j];
    }
    __syncthreads();
    least |= (uint32_t)c.bin << shift;
    room -= c.above;
    cluster.sync();                                      // the histograms have been read
  }
  const bool some = a.budget > a.n_first + a.n_last;     // else: none of the others
  // A warp's tokens of the share: above the least weight, equal to it.
  const int per = (hi - lo + kWarps * 32 - 1) / (kWarps * 32) * 32;
  const int w0 = min(hi, lo + warp * per), w1 = min(hi, w0 + per);
  auto kind = [&](int i, bool& sure, bool& equal) {      // kept for sure; kept where there is room
    const bool mid = i >= mid0 && i < mid1;
    const uint32_t k = mid && some ? key_at(i) : 0u;
    sure = i < w1 && (!mid || (some && k > least));
    equal = i < w1 && mid && some && k == least;
  };
  int gt = 0, eq = 0;
  for (int i = w0; i < w1; i += 32) {
    bool sure, equal;
    kind(i + lane, sure, equal);
    gt += __popc(__ballot_sync(0xffffffffu, sure));
    eq += __popc(__ballot_sync(0xffffffffu, equal));
  }
  if (lane == 0) { c.wsum[warp][0] = gt; c.wsum[warp][1] = eq; }
  __syncthreads();
  if (tid == 0) {
    int x = 0, y = 0;
    for (int i = 0; i < kWarps; ++i) { x += c.wsum[i][0]; y += c.wsum[i][1]; }
    c.gt = x; c.eq = y;
  }
  cluster.sync();
  int sure_before = 0, equal_before = 0;
  for (int i = 0; i < rank; ++i) { sure_before += *cluster.map_shared_rank(&c.gt, i); equal_before += *cluster.map_shared_rank(&c.eq, i); }
  for (int i = 0; i < warp; ++i) { sure_before += c.wsum[i][0]; equal_before += c.wsum[i][1]; }
  for (int i = w0; i < w1; i += 32) {
    bool sure, equal;
    kind(i + lane, sure, equal);
    const unsigned below = (1u << lane) - 1, ms = __ballot_sync(0xffffffffu, sure), me = __ballot_sync(0xffffffffu, equal);
    const int e = equal_before + __popc(me & below);
    if (sure || (equal && e < room)) kept[sure_before + __popc(ms & below) + min(e, room)] = i + lane;
    sure_before += __popc(ms);
    equal_before += __popc(me);
  }
  __threadfence();
  cluster.sync();                                        // the list is complete

  // ---------------------------------------------------------------- the move
  int64_t round = 0;
  constexpr int kRound = kCluster * kTile;
  while ((round + 1) * kRound <= keep && __ldcg(kept + (round + 1) * kRound - 1) == (round + 1) * kRound - 1) ++round;   // these stay
  uint4 x[kPieces];
  float w = 0.f;
  auto places = [&](int64_t r, int buf) {                // where the tokens of round r's places come from
    if (tid < 2 * kTile) {
      const int kv = tid / kTile, i = tid % kTile;
      const int64_t j = r * kRound + rank * kTile + i;
      int64_t from = -1;
      int b = 0;
      if (j < keep) {
        const int src = __ldcg(kept + j);
        from = page_row(p, __ldg(table + (src >> p.page_log2)), kv, g, src & in_page);
        b = scale[scale_at(from)];
      }
      int most = b;
#pragma unroll
      for (int o = 1; o < kBlock; o <<= 1) most = max(most, __shfl_xor_sync(0xffffffffu, most, o));
      c.shift[buf][kv][i] = (unsigned char)(most - b);
      c.byte[buf][kv][i] = (unsigned char)most;
      if (kv == 0) {
        c.from[buf][i] = from;
        if (from >= 0) w = mass[(((from >> p.page_log2) / (2 * G) * G + g) << p.page_log2) + (from & in_page)];
      }
    }
  };
  const int64_t to_v = (int64_t)G << p.page_log2;
  auto load = [&](int buf) {
#pragma unroll
    for (int i = 0; i < kPieces; ++i) {
      const int piece = tid + i * kThreads, token = piece >> 4, kv = piece >> 3 & 1;
      const int64_t from = c.from[buf][token];
      if (from >= 0) x[i] = *reinterpret_cast<const uint4*>(codes + (from + (kv ? to_v : 0)) * kHeadDim + 16 * (piece & 7));
    }
  };
  int buf = 0;
  if (round * kRound < keep) {
    places(round, buf);
    __syncthreads();
    load(buf);
  }
  for (; round * kRound < keep; ++round, buf ^= 1) {
    float w_now = w;
    uint4 y[kPieces];
#pragma unroll
    for (int i = 0; i < kPieces; ++i) y[i] = x[i];
    const int64_t first = round * kRound + rank * kTile;
    if (tid < kTile) {
      const int64_t j = first + tid;
      c.to[tid] = j < keep ? page_row(p, __ldg(table + (j >> p.page_log2)), 0, g, (int)(j & in_page)) : -1;
    }
    cluster.sync();                                      // every CTA has read this round's tokens
    if ((round + 1) * kRound < keep) places(round + 1, buf ^ 1);
    __syncthreads();
    if ((round + 1) * kRound < keep) load(buf ^ 1);
#pragma unroll
    for (int i = 0; i < kPieces; ++i) {
      const int piece = tid + i * kThreads, token = piece >> 4, kv = piece >> 3 & 1;
      const int64_t to = c.to[token];
      if (to < 0) continue;
      const int shift = c.shift[buf][kv][token];
      if (shift) {
        const Rescale by(shift);
        y[i] = make_uint4(by.four(y[i].x), by.four(y[i].y), by.four(y[i].z), by.four(y[i].w));
      }
      *reinterpret_cast<uint4*>(codes + (to + (kv ? to_v : 0)) * kHeadDim + 16 * (piece & 7)) = y[i];
    }
    if (tid < 2 * kTile) {
      const int kv = tid / kTile, i = tid % kTile;
      const int64_t to = c.to[i];
      if (to >= 0) {
        if ((i & (kBlock - 1)) == 0) scale[scale_at(to + (kv ? to_v : 0))] = c.byte[buf][kv][i];
        if (kv == 0) mass[(((to >> p.page_log2) / (2 * G) * G + g) << p.page_log2) + (to & in_page)] = w_now;
      }
    }
    __syncthreads();                                     // `to` and this buffer are written again
  }
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
  const int64_t longest = (((int64_t)p.max_pages << p.page_log2) + kCluster * 32 - 1) / (kCluster * 32) * 32;
  a.cache = (int)(longest < kMostCached ? longest : kMostCached);
  static std::atomic<int> smem_set[64];
  int dev = 0;
  if (cudaGetDevice(&dev) != cudaSuccess || dev < 0 || dev >= 64 || smem_set[dev].load(std::memory_order_acquire) == 0) {
    if (cudaFuncSetAttribute(paged8_evict_kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)(sizeof(Shared) + 4 * kMostCached)) != cudaSuccess)
      return -1;
    if (dev >= 0 && dev < 64) smem_set[dev].store(1, std::memory_order_release);
  }
  const unsigned heads = (unsigned)p.S * n_layers * p.G;
  return launch_pdl(paged8_evict_kernel, dim3(heads * kCluster), kThreads, sizeof(Shared) + 4 * (size_t)a.cache, st, a) ? 1 : -1;
}

}  // namespace vr
