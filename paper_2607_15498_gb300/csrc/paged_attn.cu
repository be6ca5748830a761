// Paged cache, attention of new tokens over the pages: the choice of the kernel, and the fp32 kernel.
//
// fp32: causal softmax attention in one pass over keys and values with the running maximum and sum of every row. The
// rows of a unit (paged_plan.cuh) are up to kRows (token, query head) pairs of one KV head, so a key read once serves the
// whole group. Scores of 32 keys at a time, four rows and two keys a thread; a warp's weights go through its own
// part of shared memory to the values, four rows and eight columns a thread. Keys and values are copied asynchronously,
// one buffer ahead; two CTAs an SM. Weights carry a factor `room`, a power of two that cancels and keeps the sum of as many as a
// sequence can have at 1 or below, so that no accumulator grows past the largest value.
// Bound by shared memory and the fp32 pipe alike (four columns of a score step: six 16-byte reads a thread for 32
// multiply-adds) and by the latencies of a step (shuffles, two barriers) at 16 warps an SM: 1469 new tokens of two sequences, 4 heads over
// 1, 64 us, 25 TFLOP/s. One token each of 59 sequences of up to 490, 48 heads over 8, 48 us, 1.2 TB/s: six rows of 64 are in use, so
// one warp of eight works.
// What was measured on the way, on the first: no cuts over the keys 187 us; cuts in tiles of 128 keys 84 to 99, in steps of 32
// with the next unit taken at the start of one 115, in its last step 64. 64 rows by 128 threads with 8 x 4 scores each:
// 90 us at tiles of 128, not measured in steps of 32. Packed products change 1 %, a prefetch to L2 nothing, and units of at most 8
// rows with the keys shared among the warps take 43 us on the second, but 5 to 12 % more on small steps.
#include <math.h>

#include <atomic>

#include "common.cuh"
#include "paged.h"
#include "paged_plan.cuh"

namespace vr {

namespace {

constexpr int kThreads = 256;
constexpr int kRows = 64, kStep = kKeysF32;      // keys of a step
constexpr float kOverhead = 2.f;           // of a unit, in steps, as the plan counts it: 1 to 8 give the chunk the same 64 us, the
                                           // steps of 59 sequences 50, 47, 48, 51 at 1, 2, 4, 8
constexpr int kPitch = kHeadDim + 4;       // floats of a query or key row: 16-byte reads of 8 rows fall on 32 banks
constexpr int kPPitch = kStep + 4;

struct Smem {
  float q[kRows][kPitch];
  float k[2][kStep][kPitch];
  float v[2][kStep][kHeadDim];
  float p[kRows][kPPitch];
  PlanSums plan;
  Unit unit;
  int seq, next;
};

__device__ __forceinline__ float4 get4(const float* s) { return *reinterpret_cast<const float4*>(s); }

__global__ void __launch_bounds__(kThreads, 2)
paged_attn_f32_kernel(Paged p, const float* __restrict__ pool, const float* __restrict__ q, float* __restrict__ out,
                      int32_t* dev_status, Header* header, float* __restrict__ part, int part_rows, int max_parts, int grp, float scale,
                      float room) {
  extern __shared__ __align__(16) unsigned char raw[];
  Smem& sm = *reinterpret_cast<Smem*>(raw);
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, H = p.G * grp, C = gridDim.x;
  const int tq = kRows / grp;               // tokens of a block
  const int ty = tid >> 4, tx = tid & 15;
  pdl_trigger();
  if (tid < kCand) { sm.plan.units[tid] = 0; sm.plan.split[tid] = 0; sm.plan.chunk[tid] = 0; }
  __syncthreads();
  pdl_wait();
  const int open = blockIdx.x == 0 && tid == 0 ? header->open : 0;   // by a call whose merge did not run, or runs still
  int longest;
  const float weight = plan_weight<kStep>(p, tq, lane, longest);
  const int cand = plan_candidate(weight, longest, C, lane);
  plan_add<kStep>(p, sm.plan, tq, cand, warp, kThreads / 32, lane);
  __syncthreads();
  int run, units, parts;
  plan_choose(sm.plan, weight, cand, C, max_parts, kOverhead, lane, run, units, parts);
  if (blockIdx.x == 0) {
    if (tid == 0) {
      if (open) raise_status(dev_status, VARRATE_ERR_CORRUPT);
      header->run = run; header->units = units; header->parts = parts; header->open = 1;
    }
    for (int s = tid; s < p.S; s += kThreads) {
      SeqRange r;
      if (!seq_range(p, s, r)) raise_status(dev_status, VARRATE_ERR_CORRUPT);
    }
  }
  Walk<kStep> w;
  if (warp == 0) w.load(p, tq, run, lane);
  int u = blockIdx.x;
  while (u < units) {
    // the unit: found by one warp
    if (warp == 0) {
      Unit x;
      const int s = w.find(p, tq, tq, run, u, lane, x);
      if (lane == 0) {
        sm.unit = x;
        sm.seq = s;
      }
    }
    __syncthreads();
    const Unit x = sm.unit;
    const int32_t* table = p.table + (int64_t)sm.seq * p.max_pages;
    const int rows = x.ntok * grp, end = min(x.pos0 + x.ntok, x.t1 * kStep), k_first = x.t0 * kStep;
    const float* qb = q + ((int64_t)x.row0 * H + (int64_t)x.g * grp) * kHeadDim;
    if (k_first >= end) {                     // the block ends before this run of keys
      if (tid == 0) sm.next = take_unit(header, C, units);
      __syncthreads();
      u = sm.next;
      continue;
    }
    // asynchronous copy of 32 keys and values from `k0` on: 4 rows of each a warp; past the end: zeros
    auto fetch = [&](int k0, int buf) {
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const int key = warp * 4 + i, t = k0 + key;
        int page = -1;
        if (t < end) {
          page = __ldg(table + (t >> p.page_log2));
          if (page < 0 || page >= p.n_pages) { raise_status(dev_status, VARRATE_ERR_CORRUPT); page = -1; }
        }
        const float* src = page < 0 ? pool : pool + page_row(p, page, 0, x.g, t & ((1 << p.page_log2) - 1)) * kHeadDim + lane * 4;
        const int64_t to_v = page < 0 ? 0 : ((int64_t)p.G << p.page_log2) * kHeadDim;
        cp_async16(smem_addr(&sm.k[buf][key][lane * 4]), src, page < 0 ? 0 : 16);
        cp_async16(smem_addr(&sm.v[buf][key][lane * 4]), src + to_v, page < 0 ? 0 : 16);
      }
      cp_async_commit();
    };
    fetch(k_first, 0);
    for (int i = tid; i < kRows * 32; i += kThreads) {
      const int row = i >> 5, c = (i & 31) * 4;
      float4 v = make_float4(0.f, 0.f, 0.f, 0.f);
      if (row < rows) v = load4(qb + ((int64_t)(row / grp) * H + row % grp) * kHeadDim + c);
      *reinterpret_cast<float4*>(&sm.q[row][c]) = make_float4(v.x * scale, v.y * scale, v.z * scale, v.w * scale);
    }
    int sees[4];                              // keys that the thread's rows see
#pragma unroll
    for (int i = 0; i < 4; ++i) sees[i] = x.pos0 + min((4 * ty + i) / grp, x.ntok - 1) + 1;
    float m[4], l[4], o[4][8];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      m[i] = -INFINITY;
      l[i] = 0.f;
#pragma unroll
      for (int j = 0; j < 8; ++j) o[i][j] = 0.f;
    }
    int buf = 0, next = 0;
    for (int k0 = k_first; k0 < end; k0 += kStep, buf ^= 1) {   // (a warp has 8 of the rows)
      cp_async_wait<0>();
      __syncthreads();                        // these keys are there, the other buffer is free
      if (k0 + kStep < end) fetch(k0 + kStep, buf ^ 1);
      else if (tid == 0) next = take_unit(header, C, units);   // not earlier: others may be free before this CTA
      if (8 * warp >= rows) continue;         // no row of this warp's
      float s[4][2] = {};
#pragma unroll 8
      for (int d = 0; d < kHeadDim; d += 4) {
        float4 a[4], b[2];
#pragma unroll
        for (int i = 0; i < 4; ++i) a[i] = get4(&sm.q[4 * ty + i][d]);
#pragma unroll
        for (int j = 0; j < 2; ++j) b[j] = get4(&sm.k[buf][tx + 16 * j][d]);
#pragma unroll
        for (int i = 0; i < 4; ++i)
#pragma unroll
          for (int j = 0; j < 2; ++j)
            s[i][j] = fmaf(a[i].x, b[j].x, fmaf(a[i].y, b[j].y, fmaf(a[i].z, b[j].z, fmaf(a[i].w, b[j].w, s[i][j]))));
      }
#pragma unroll
      for (int i = 0; i < 4; ++i) {
#pragma unroll
        for (int j = 0; j < 2; ++j)
          if (k0 + tx + 16 * j >= sees[i]) s[i][j] = -INFINITY;
        float mx = fmaxf(s[i][0], s[i][1]);
#pragma unroll
        for (int w2 = 8; w2 > 0; w2 >>= 1) mx = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, w2));
        const float mn = fmaxf(m[i], mx), ref = mn == -INFINITY ? 0.f : mn;   // no finite score yet: weights 0
        const float f = exp2f((m[i] - ref) * kLog2e);
        m[i] = mn;
        float sum = 0.f;
#pragma unroll
        for (int j = 0; j < 2; ++j) {
          const float e = exp2f((s[i][j] - ref) * kLog2e) * room;
          sm.p[4 * ty + i][tx + 16 * j] = e;
          sum += e;
        }
        l[i] = l[i] * f + sum;
#pragma unroll
        for (int j = 0; j < 8; ++j) o[i][j] *= f;
      }
      __syncwarp();                           // a warp's weights are its own
      const bool cut = k0 + kStep > x.pos0 + 1;   // some row does not see all of these keys: weight 0 is no product there
#pragma unroll 2
      for (int key = 0; key < kStep; key += 4) {
        float e[4][4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const float4 y = get4(&sm.p[4 * ty + i][key]);
          e[i][0] = y.x; e[i][1] = y.y; e[i][2] = y.z; e[i][3] = y.w;
        }
#pragma unroll
        for (int kk = 0; kk < 4; ++kk) {
          const float4 v0 = get4(&sm.v[buf][key + kk][4 * tx]), v1 = get4(&sm.v[buf][key + kk][64 + 4 * tx]);
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            if (cut && k0 + key + kk >= sees[i]) continue;
            const float a = e[i][kk];
            o[i][0] = fmaf(a, v0.x, o[i][0]); o[i][1] = fmaf(a, v0.y, o[i][1]);
            o[i][2] = fmaf(a, v0.z, o[i][2]); o[i][3] = fmaf(a, v0.w, o[i][3]);
            o[i][4] = fmaf(a, v1.x, o[i][4]); o[i][5] = fmaf(a, v1.y, o[i][5]);
            o[i][6] = fmaf(a, v1.z, o[i][6]); o[i][7] = fmaf(a, v1.w, o[i][7]);
          }
        }
      }
      __syncwarp();
    }
    float* ob = out + ((int64_t)x.row0 * H + (int64_t)x.g * grp) * kHeadDim;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int row = 4 * ty + i;
      float sum = l[i];
#pragma unroll
      for (int w2 = 8; w2 > 0; w2 >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, w2);
      if (row >= rows) continue;
      const bool whole = x.slot < 0;
      const float f = !whole ? 1.f : sum == 0.f ? 0.f : 1.f / sum;
      const int64_t pr = (int64_t)x.slot * part_rows + row;
      float* d = whole ? ob + ((int64_t)(row / grp) * H + row % grp) * kHeadDim : part + pr * kHeadDim;
      *reinterpret_cast<float4*>(d + 4 * tx) = make_float4(o[i][0] * f, o[i][1] * f, o[i][2] * f, o[i][3] * f);
      *reinterpret_cast<float4*>(d + 64 + 4 * tx) = make_float4(o[i][4] * f, o[i][5] * f, o[i][6] * f, o[i][7] * f);
      if (!whole && tx == 0)                  // references of partials are in log2 units; a row without a weight has no say
        reinterpret_cast<float2*>(part + (int64_t)max_parts * part_rows * kHeadDim)[pr] = make_float2(sum == 0.f ? -INFINITY : m[i] * kLog2e, sum);
    }
    if (tid == 0) sm.next = next;
    __syncthreads();                          // queries, buffers and the unit are free
    u = sm.next;
  }
}

}  // namespace

size_t paged_attn_ws_bytes(const Paged& p, int group, int num_sms) {
  return p.dtype == VARRATE_F32 ? paged_part_bytes(p, group, kRows / group, 2 * num_sms) : paged_attn_tc_ws_bytes(p, group, num_sms);
}

int launch_paged_attn(const Paged& p, int layer, int group, const void* q, void* out, int32_t* dev_status, void* ws,
                      int num_sms, cudaStream_t st) {
  if (p.dtype != VARRATE_F32) return launch_paged_attn_tc(p, layer, group, q, out, dev_status, ws, num_sms, st);
  static std::atomic<int> smem_set[64];
  int dev = 0;
  if (cudaGetDevice(&dev) != cudaSuccess || dev < 0 || dev >= 64 || smem_set[dev].load(std::memory_order_acquire) == 0) {
    if (cudaFuncSetAttribute(paged_attn_f32_kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)sizeof(Smem)) != cudaSuccess)
      return -1;
    if (dev >= 0 && dev < 64) smem_set[dev].store(1, std::memory_order_release);
  }
  const int tq = kRows / group, ctas = 2 * num_sms;
  Header* header = static_cast<Header*>(ws);
  float* part = reinterpret_cast<float*>(static_cast<unsigned char*>(ws) + kHeaderBytes);
  const float* pool = reinterpret_cast<const float*>(p.pool) + (int64_t)layer * p.layer_rows * kHeadDim;
  int bits = 0;
  while (bits < 31 && ((int64_t)1 << bits) < ((int64_t)p.max_pages << p.page_log2)) ++bits;   // keys of a sequence: 2^bits at most
  if (!launch_pdl(paged_attn_f32_kernel, dim3(ctas), kThreads, sizeof(Smem), st, p, pool, (const float*)q, (float*)out, dev_status,
                  header, part, paged_part_rows(p, group, tq), paged_max_parts(ctas), group, 1.f / sqrtf((float)kHeadDim),
                  ldexpf(1.f, -bits)))
    return -1;
  return launch_paged_merge(p, group, out, dev_status, header, part, tq, tq, ctas, st) < 0 ? -1 : 2;
}

}  // namespace vr
