// Paged cache in 8 bits, attention weight of every cached token: mass[u] += sum over rows that see u of 2^(score - log2 e lse).
//
// The products are those of the attention of few rows (paged8_mma.cuh): a warp takes 16 keys and eight rows at a time, every
// row that sees a key, and adds up in registers, so a token's sum has one order. The steps of 16 keys of all sequences and KV heads
// are one line that the warps share equally.
//
// Bound by memory: single tokens on eight sequences of 32768, 50 us for 285 MB (keys, scales, and 8 bytes a token and head), 5.7 TB/s
// (0.84 of a copy). Three steps in flight a warp, sixteen warps an SM (96 KB); 70 us in a form whose registers spilled.
#include <float.h>
#include <math.h>

#include <atomic>

#include <cudaTypedefs.h>

#include "common.cuh"
#include "paged.h"
#include "paged8.h"
#include "paged8_mma.cuh"

namespace vr {

bool make_tmap_rows_u8(CUtensorMap* map, const void* base, uint64_t rows, uint32_t box_rows);

namespace {

constexpr int kThreads = 256, kWarps = kThreads / 32, kCtas = 2;
constexpr int kRows = 8;
constexpr int kStages = 3, kStepBytes = 16 * kHeadDim;              // a warp's steps in flight

struct Shared {
  unsigned char ring[kWarps][kStages][kStepBytes];
  uint64_t full[kWarps][kStages];
};

// Steps of 16 keys of a sequence, all KV heads; 0 where it has no new tokens, or more than `few`.
__device__ __forceinline__ int64_t steps_of(const Paged& p, int s, int few, SeqRange& r) {
  if (s >= p.S || !seq_range(p, s, r) || r.n == 0 || r.n > few) return 0;
  return (int64_t)((r.len + 15) >> 4) * p.G;
}

__global__ void __launch_bounds__(kThreads, kCtas)
paged8_mass_kernel(const __grid_constant__ CUtensorMap tmap, Paged p, const unsigned char* __restrict__ scale,
                   float* __restrict__ mass, const __nv_bfloat16* __restrict__ q, const float* __restrict__ lse,
                   int32_t* __restrict__ dev_status, int grp, int few, float scale_log2) {
  extern __shared__ __align__(1024) unsigned char smem[];
  Shared& c = *reinterpret_cast<Shared*>(smem);
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, g8 = lane >> 2, t4 = lane & 3, H = p.G * grp, tq = kRows / grp;
  if (lane == 0) {                                                  // (a warp's own)
    for (int i = 0; i < kStages; ++i) mbar_init(&c.full[warp][i], 1);
    fence_mbar_init();
  }
  __syncwarp();
  pdl_trigger();
  pdl_wait();
  int64_t total = 0;
  for (int s = lane; s < p.S; s += 32) {
    SeqRange r;
    total += steps_of(p, s, few, r);
    if (blockIdx.x == 0 && tid < 32 && !seq_range(p, s, r)) raise_status(dev_status, VARRATE_ERR_CORRUPT);
  }
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) total += __shfl_xor_sync(0xffffffffu, total, o);
  const int64_t warps = (int64_t)gridDim.x * kWarps, id = (int64_t)blockIdx.x * kWarps + warp;
  int64_t at = total * id / warps;
  const int64_t stop = total * (id + 1) / warps;
  if (at >= stop) return;
  uint32_t stage = 0, phase = 0;
  bool ok = true;

  // the sequence of step `at`: 32 sequences at a time
  int s0 = 0;
  int64_t before = 0, incl = 0;
  SeqRange r;
  auto scan = [&]() {
    incl = steps_of(p, s0 + lane, few, r);
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const int64_t y = __shfl_up_sync(0xffffffffu, incl, o);
      if (lane >= o) incl += y;
    }
  };
  scan();
  while (at < stop) {
    while (at >= before + __shfl_sync(0xffffffffu, incl, 31)) {
      before += __shfl_sync(0xffffffffu, incl, 31);
      s0 += 32;
      scan();
    }
    const int l = __ffs(__ballot_sync(0xffffffffu, at < before + incl)) - 1, s = s0 + l;
    const int len = __shfl_sync(0xffffffffu, r.len, l), n = __shfl_sync(0xffffffffu, r.n, l), row0 = __shfl_sync(0xffffffffu, r.row0, l);
    const int per = (len + 15) >> 4;                                // steps of a head
    const int64_t off = at - (before + __shfl_sync(0xffffffffu, incl, l) - (int64_t)per * p.G);
    const int g = (int)(off / per), st0 = (int)(off - (int64_t)g * per);
    const int st1 = (int)min((int64_t)per, st0 + (stop - at));
    const int32_t* table = p.table + (int64_t)s * p.max_pages;
    Steps steps{p, scale, table, dev_status, g, st0, 1, st1 - st0};
    steps.start(lane);
    auto request = [&](int i, uint32_t to) {                        // step i into stage `to`
      const int row = steps.row(steps.page(i), i);
      if (lane == 0) {
        mbar_arrive_expect_tx(&c.full[warp][to], kStepBytes);
        tma_load_2d(smem_addr(c.ring[warp][to]), &tmap, 0, row, &c.full[warp][to]);
      }
    };
    uint32_t ahead = stage;
    for (int i = 0; i < min(steps.n, kStages); ++i) {
      request(i, ahead);
      ahead = ahead + 1 == kStages ? 0 : ahead + 1;
    }
    struct Rows {
      QueryFrags q;
      float e0, e1;                                                 // log2 e lse of rows 2 t4, 2 t4 + 1; infinity where one adds nothing
      int sees0, sees1;                                             // keys that they see
    };
    auto load_rows = [&](int b, Rows& x) {                          // eight rows: tokens b * tq ..
      const int ntok = max(0, min(tq, n - b * tq)), rows = ntok * grp, first = row0 + b * tq, pos0 = len - n + b * tq;
      x.q.load(q + ((int64_t)(first + g8 / grp) * H + g * grp + g8 % grp) * kHeadDim, g8 < rows, scale_log2, lane);
      auto less = [&](int i) {
        if (i >= rows) return INFINITY;
        const float y = __ldg(lse + (int64_t)(first + i / grp) * H + g * grp + i % grp);
        return fabsf(y) < INFINITY ? y * kLog2e : INFINITY;
      };
      x.e0 = less(2 * t4);
      x.e1 = less(2 * t4 + 1);
      x.sees0 = pos0 + 2 * t4 / grp + 1;
      x.sees1 = pos0 + (2 * t4 + 1) / grp + 1;
    };
    Rows rows[2];
    load_rows(0, rows[0]);
    load_rows(1, rows[1]);
    const int blocks = (n + tq - 1) / tq;                           // two stay in registers
    int i = 0;
    for (; i < steps.n; ++i) {
      ok = warp_wait(&c.full[warp][stage], phase);
      if (!ok) break;
      uint4 kq[4];
      read_keys(c.ring[warp][stage], lane, kq);
      const int page = steps.page(i), key0 = (st0 + i) << 4;
      const float f = __uint_as_float((steps.bytes(i) & 0xff) << 23);
      float w0 = 0.f, w1 = 0.f;                                     // of keys g8, g8 + 8
      auto add = [&](const Rows& x) {
        float sc[4];
        key_scores(kq, x.q, sc);
        const float f0 = fminf(x.q.f0 * f, FLT_MAX), f1 = fminf(x.q.f1 * f, FLT_MAX);
        const int a = key0 + g8, d = a + 8;
        if (a < x.sees0 && x.e0 < INFINITY) w0 += fast_exp2(sc[0] * f0 - x.e0);
        if (a < x.sees1 && x.e1 < INFINITY) w0 += fast_exp2(sc[1] * f1 - x.e1);
        if (d < x.sees0 && x.e0 < INFINITY) w1 += fast_exp2(sc[2] * f0 - x.e0);
        if (d < x.sees1 && x.e1 < INFINITY) w1 += fast_exp2(sc[3] * f1 - x.e1);
      };
      add(rows[0]);
#pragma unroll 1
      for (int b = 1; b < blocks; ++b) {
        if (blocks > 2) load_rows(b, rows[1]);
        add(rows[1]);
      }
      __syncwarp();                                                 // the tile has been read
      if (i + kStages < steps.n) request(i + kStages, stage);
#pragma unroll
      for (int o = 1; o < 4; o <<= 1) {
        w0 += __shfl_xor_sync(0xffffffffu, w0, o);
        w1 += __shfl_xor_sync(0xffffffffu, w1, o);
      }
      // one addition to a token in a call: the order is no matter
      if (t4 < 2 && page >= 0 && key0 + g8 + 8 * t4 < len) atomicAdd(mass + mass_at(p, page, g, steps.in_page(i) + g8 + 8 * t4), t4 ? w1 : w0);
      steps.done(i, lane);
      if (++stage == kStages) { stage = 0; phase ^= 1; }
    }
    if (!ok) {                                                      // no copy is in flight when the block ends
      for (int j = i; j < min(steps.n, i + kStages); ++j) {
        warp_wait(&c.full[warp][stage], phase);
        if (++stage == kStages) { stage = 0; phase ^= 1; }
      }
      raise_status(dev_status, VARRATE_ERR_TIMEOUT);
      break;
    }
    at += st1 - st0;
  }
}

}  // namespace

int launch_paged8_mass(const Paged8& c, int layer, int group, const void* q, const float* lse, int32_t* dev_status,
                       int num_sms, cudaStream_t st) {
  const Paged& p = c.p;
  const bool many = p.T > few_tokens(p, group);                        // else no sequence can have more
  if (many && launch_paged8_mass_tc(c, layer, group, q, lse, dev_status, num_sms, st) < 0) return -1;
  CUtensorMap tmap;
  if (!make_tmap_rows_u8(&tmap, p.pool + (int64_t)layer * p.layer_rows * kHeadDim, (uint64_t)p.layer_rows, 16)) return -1;
  static std::atomic<int> smem_set[64];
  int dev = 0;
  if (cudaGetDevice(&dev) != cudaSuccess || dev < 0 || dev >= 64 || smem_set[dev].load(std::memory_order_acquire) == 0) {
    if (cudaFuncSetAttribute(paged8_mass_kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)sizeof(Shared)) != cudaSuccess) return -1;
    if (dev >= 0 && dev < 64) smem_set[dev].store(1, std::memory_order_release);
  }
  if (!launch_pdl(paged8_mass_kernel, dim3(kCtas * num_sms), kThreads, sizeof(Shared), st, tmap, p,
                  c.scale + (int64_t)layer * (p.layer_rows >> kBlockLog2), c.mass + (int64_t)layer * (p.layer_rows / 2),
                  (const __nv_bfloat16*)q, lse, dev_status, group, few_tokens(p, group), kLog2e / sqrtf((float)kHeadDim)))
    return -1;
  return many ? 2 : 1;
}

}  // namespace vr
