// Paged cache in 8 bits, attention weight of every cached token: mass[u] += sum over rows that see u of 2^(score - log2 e lse).
//
// The products are those of the attention of few rows (paged8_mma.cuh): a warp takes 16 keys and eight rows at a time, every
// row that sees a key, and adds up in registers, so a token's sum has one order. The steps of 16 keys of all sequences and KV heads
// are one line that the warps share equally. Bound by memory for single tokens (keys and 8 bytes a token and head).
#include <float.h>
#include <math.h>

#include "common.cuh"
#include "paged.h"
#include "paged8.h"
#include "paged8_mma.cuh"

namespace vr {

namespace {

constexpr int kThreads = 256, kWarps = kThreads / 32, kCtas = 2;
constexpr int kRows = 8;

// Steps of 16 keys of a sequence, all KV heads; 0 where it has no new tokens.
__device__ __forceinline__ int64_t steps_of(const Paged& p, int s, SeqRange& r) {
  if (s >= p.S || !seq_range(p, s, r) || r.n == 0) return 0;
  return (int64_t)((r.len + 15) >> 4) * p.G;
}

__global__ void __launch_bounds__(kThreads, kCtas)
paged8_mass_kernel(Paged p, const unsigned char* __restrict__ codes, const unsigned char* __restrict__ scale,
                   float* __restrict__ mass, const __nv_bfloat16* __restrict__ q, const float* __restrict__ lse,
                   int32_t* __restrict__ dev_status, int grp, float scale_log2) {
  const int tid = threadIdx.x, lane = tid & 31, g8 = lane >> 2, t4 = lane & 3, H = p.G * grp, tq = kRows / grp;
  pdl_trigger();
  pdl_wait();
  int64_t total = 0;
  for (int s = lane; s < p.S; s += 32) {
    SeqRange r;
    total += steps_of(p, s, r);
    if (blockIdx.x == 0 && tid < 32 && !seq_range(p, s, r)) raise_status(dev_status, VARRATE_ERR_CORRUPT);
  }
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) total += __shfl_xor_sync(0xffffffffu, total, o);
  const int64_t warps = (int64_t)gridDim.x * kWarps, id = (int64_t)blockIdx.x * kWarps + (tid >> 5);
  int64_t at = total * id / warps;
  const int64_t stop = total * (id + 1) / warps;
  if (at >= stop) return;
  const int in_page = (1 << p.page_log2) - 1;

  // the sequence of step `at`: 32 sequences at a time
  int s0 = 0;
  int64_t before = 0, incl = 0;
  SeqRange r;
  auto scan = [&]() {
    incl = steps_of(p, s0 + lane, r);
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
    const int blocks = (int)((unsigned)(n + tq - 1) / (unsigned)tq);
    QueryFrags qf;
    float e0 = 0.f, e1 = 0.f;
    int sees0 = 0, sees1 = 0;
    auto load_rows = [&](int b) {                                   // eight rows: tokens b * tq ..
      const int ntok = min(tq, n - b * tq), rows = ntok * grp, first = row0 + b * tq;
      qf.load(q + ((int64_t)(first + g8 / grp) * H + g * grp + g8 % grp) * kHeadDim, g8 < rows, scale_log2, lane);
      auto less = [&](int i) {                                      // log2 e lse of row i; infinity where it adds nothing
        if (i >= rows) return INFINITY;
        const float y = __ldg(lse + (int64_t)(first + i / grp) * H + g * grp + i % grp);
        return fabsf(y) < INFINITY ? y * kLog2e : INFINITY;
      };
      e0 = less(2 * t4);
      e1 = less(2 * t4 + 1);
      const int pos0 = len - n + b * tq;
      sees0 = pos0 + 2 * t4 / grp + 1;
      sees1 = pos0 + (2 * t4 + 1) / grp + 1;
    };
    auto row_of = [&](int step) {
      int page = __ldg(table + ((step << 4) >> p.page_log2));
      if (page < 0 || page >= p.n_pages) { raise_status(dev_status, VARRATE_ERR_CORRUPT); return (int64_t)-1; }
      return page_row(p, page, 0, g, (step << 4) & in_page);
    };
    if (blocks == 1) load_rows(0);
    for (int st = st0; st < st1; ++st) {
      const int64_t row = row_of(st);
      const int key0 = st << 4;
      if (row < 0) continue;
      uint4 kq[4];
      const unsigned char* src = codes + row * kHeadDim + 16 * t4;
#pragma unroll
      for (int i = 0; i < 4; ++i) kq[i] = __ldg(reinterpret_cast<const uint4*>(src + (g8 + 8 * (i >> 1)) * kHeadDim + 64 * (i & 1)));
      const float f = __uint_as_float((uint32_t)__ldg(scale + scale_at(row)) << 23);
      float w0 = 0.f, w1 = 0.f;                                     // of keys g8, g8 + 8
      // the first block whose last token sees the first key
      for (int b = max(0, (int)((unsigned)max(0, key0 - (len - n)) / (unsigned)tq)); b < blocks; ++b) {
        if (blocks > 1) load_rows(b);
        float sc[4];
        key_scores(kq, qf, sc);
        const float f0 = fminf(qf.f0 * f, FLT_MAX), f1 = fminf(qf.f1 * f, FLT_MAX);
        const int a = key0 + g8, c = a + 8;
        if (a < sees0 && e0 < INFINITY) w0 += fast_exp2(sc[0] * f0 - e0);
        if (a < sees1 && e1 < INFINITY) w0 += fast_exp2(sc[1] * f1 - e1);
        if (c < sees0 && e0 < INFINITY) w1 += fast_exp2(sc[2] * f0 - e0);
        if (c < sees1 && e1 < INFINITY) w1 += fast_exp2(sc[3] * f1 - e1);
      }
#pragma unroll
      for (int i = 1; i < 4; i <<= 1) {
        w0 += __shfl_xor_sync(0xffffffffu, w0, i);
        w1 += __shfl_xor_sync(0xffffffffu, w1, i);
      }
      if (t4 < 2) {
        const int key = key0 + g8 + 8 * t4;
        float* m = mass + (((row >> p.page_log2) / (2 * p.G) * p.G + g) << p.page_log2) + (key & in_page);
        if (key < len) *m += t4 ? w1 : w0;
      }
    }
    at += st1 - st0;
  }
}

}  // namespace

int launch_paged8_mass(const Paged8& c, int layer, int group, const void* q, const float* lse, int32_t* dev_status,
                       int num_sms, cudaStream_t st) {
  const Paged& p = c.p;
  return launch_pdl(paged8_mass_kernel, dim3(kCtas * num_sms), kThreads, 0, st, p,
                    p.pool + (int64_t)layer * p.layer_rows * kHeadDim, c.scale + (int64_t)layer * (p.layer_rows >> kBlockLog2),
                    c.mass + (int64_t)layer * (p.layer_rows / 2), (const __nv_bfloat16*)q, lse, dev_status, group,
                    kLog2e / sqrtf((float)kHeadDim))
             ? 1 : -1;
}

}  // namespace vr
