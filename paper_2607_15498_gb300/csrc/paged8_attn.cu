// Paged cache in 8 bits, attention of few new tokens: codes go from memory to registers and, as they are, into tensor-core
// products of fp16 fragments (mma.sync).
//
// A row is a (token, query head) pair of one KV head; a CTA works for a block of at most 8 rows, a warp on steps of 16 keys, which
// share a scale. Per step, transposed so that 8 rows fill the products:
//   S^T[key][row] = K[key][.] Q[row][.]     8 products of 16 keys x 8 rows x 16 elements,
//   O^T[element][row] += V^T[element][key] P^T[key][row]     8 products of 16 elements x 8 rows x 16 keys.
// An e4m3 code is exact in fp16 and two are expanded by one instruction. Which element of a head an operand's index means is
// free as long as both operands agree, so that a lane takes 16 bytes of a key (or of four keys' values) as they stand in the page.
//   queries  x 2^n with the largest element of a row in [2^14, 2^15): exact in fp16 down to 2^-38 of it;
//   scores   x (scale of the block) x (2^-n log2 e / sqrt(d)) in fp32;
//   weights  p x 2^(7 + b - u) in fp16, b the scale byte of the step's values and u that of the accumulator, which is
//            in units of 2^(u - 127), u the largest b so far.
// A row's reference (log2) stands where fp16 has its places for the weights of most keys: those between 2^-24
// and 2^8 of it go in one product a step (2^-17 to 2^15 as stored: half a step of fp16 is 2^-8 of the smallest, no more than bf16's
// would be). A step with others moves the reference where that takes them in, and gives what is left products of its own, times what
// brings the largest to 2^14, as often as it takes: what a heavy token without a value leaves to the others is not lost. The largest weight
// of such a band, and of the step that sets a reference first, is a power of two as stored, not rounded: where one token has most of the
// weight the output is its value to fp32 (0.0005 of its size from the plain form's for 0.0011 on the batch below). The sums, in fp32, may grow to 2^72 and their range below; what goes is values below 2^-100 or so of the largest block's.
// How far a score is from the reference is their difference: the sum of a large reference and 8 may round up to 16 above it.
// Units of work, partials and their merge are those of the uncompressed cache's attention (paged_plan.cuh). Codes come by TMA into
// a ring of each warp's own, two steps of keys and values in flight a warp and sixteen warps an SM: 128 KB.
//
// Bound by memory for batches: eight sequences of 32768 tokens 93 us with the merge, 538 MB at 5.8 TB/s (0.85 of a copy), 98 where one key
// in 200 is four times as long as the others and one step in twelve so takes products in several bands. By latency for
// short ones: one sequence of 900 tokens 10.4 us, of which the plan is 2.5, the first step 2 and the merge 2.5.
// On the way, that batch: three stages of one CTA an SM 95 us, the next step's codes in registers 133, sixteen warps in one CTA 100.
// One product a step from the largest score on, light weights lost, 91.5; those in bf16 products beside it 116; every step in bands 112.
// Where sequences of the batch may have many new tokens, the kernel on tcgen05 is launched behind this one and waits for it as any kernel
// for the one before: its barriers and TMEM are set up by then. (The other order, this one beginning on the SMs that the other
// has left, is not one that a kernel may have without a wait of its own; it took 64.2 us for 67.2 on a chunk beside 23 single tokens, 148
// for 138 on one beside 32.)
#include <float.h>
#include <math.h>

#include <atomic>

#include <cudaTypedefs.h>

#include "common.cuh"
#include "paged.h"
#include "paged8.h"
#include "paged8_mma.cuh"
#include "paged_plan.cuh"

namespace vr {

bool make_tmap_rows_u8(CUtensorMap* map, const void* base, uint64_t rows, uint32_t box_rows);

namespace {

constexpr int kThreads = 256, kWarps = kThreads / 32, kCtas = 2;
constexpr int kRows = 8, kKeys = kKeysBf16;
constexpr float kOverhead = 8.f;             // of a unit, in key tiles, as the plan counts it
constexpr int kUp = 7;                       // weights are stored times 2^kUp
constexpr float kSlack = 8.f, kLow = 17.f + kUp;   // what scores may be above and below the reference for one product a step (log2)
constexpr float kMost = 0x1p15f, kLeast = 0x1p-17f;   // the same of a weight as it is stored
constexpr float kFar = 72.f;                 // how far weights and sums of a row may grow (log2)
constexpr int kBands = 10;                   // bands of 2^31 that hold all weights of fp32

constexpr int kStages = 2, kStepBytes = 16 * kHeadDim * 2;           // a warp's steps in flight: keys, then values
struct Shared {
  union {
    unsigned char ring[kWarps][kStages][kStepBytes];
    float o[kWarps][kRows][kHeadDim + 4];                           // at the end of a unit
  };
  uint64_t full[kWarps][kStages];
  PlanSums plan;
  SeqUnit unit;
  int err;
  float m[kWarps][kRows], l[kWarps][kRows];
  int u[kWarps];
};
static_assert(kCtas * (sizeof(Shared) + 2048) <= 228 * 1024, "shared memory of an SM");

// Values of a step with rows that do not see all of its keys: those past the batch's tokens are zeroed; NaN codes of keys that
// only a part of the rows sees are zeroed and returned as bits, 16 codes a key.
__device__ __forceinline__ bool take_nan(uint4& v, uint32_t& bits) {
  uint32_t* w = reinterpret_cast<uint32_t*>(&v);
  bits = 0;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const uint32_t n = __vcmpeq4(w[i] & 0x7f7f7f7fu, 0x7f7f7f7fu);
    w[i] &= ~n;
    bits |= ((n & 1) | (n >> 7 & 2) | (n >> 14 & 4) | (n >> 21 & 8)) << (4 * i);
  }
  return bits != 0;
}

// A row's reference m after a step whose weights fp16 has not the places for as it stands: the factor for what the row has added up, a
// power of two but for a rounding of m. x, y: the lane's two scores of the row, whose others are in the lanes of the same four; l: the lane's sum. low: what
// scores may be below the reference, less where the block's values are smaller than the accumulator's unit.
__device__ __forceinline__ float move_reference(float& m, float l, float x, float y, float low) {
  float a = fmaxf(x, y), b = fminf(x == -INFINITY ? INFINITY : x, y == -INFINITY ? INFINITY : y);   // of the scores that count
#pragma unroll
  for (int i = 4; i < 32; i <<= 1) {
    a = fmaxf(a, __shfl_xor_sync(0xffffffffu, a, i));
    b = fminf(b, __shfl_xor_sync(0xffffffffu, b, i));
    l = fmaxf(l, __shfl_xor_sync(0xffffffffu, l, i));
  }
  if (a == -INFINITY) return 1.f;
  // the step's scores in the middle of what there is room for where they fit in, else the largest near its end
  const bool narrow = a - b <= kSlack + kLow - 2.f;
  const float below = ceilf(narrow ? 0.5f * (a - b - (kLow - kSlack)) : kSlack - 1.f);   // of the largest: the new reference
  if (l == 0.f) {                                                   // nothing added up yet: the largest weight is a power of two
    m = a - below;
    return 1.f;
  }
  float by = 0.f;
  if (a - m > kFar) by = floorf(a - m - (kFar - kSlack));           // sums would come near fp32's end
  else if (a - m > kSlack ? narrow : b - m < low) by = fmaxf(narrow ? floorf(a - m - below) : fminf(floorf(a - m - below), 0.f), -floorf(fmaxf(kFar - __log2f(l), 0.f)));
  const float was = m;
  m += by;
  return fast_exp2(was - m);
}

// At the end of a unit: the sum l of a row to [1, 2), its reference m up by as much, as the references of warps and units are compared,
// where a rounding of m is not more than one of its scores was (and stays small: scores past 2^12 may be exact and near each other); the factor for the row's values, which are times 2^kUp.
__device__ __forceinline__ float settle(float& m, float& l) {
  if (l == 0.f) m = -INFINITY;                                      // no score: no say in a merge
  const int e = (int)(__float_as_uint(l) >> 23) - 127;
  const float up = m + (float)e;
  if (!(l > 0.f && e <= 126 && fabsf(up - m - (float)e) <= 0x1p-12f)) return 1.f / (1 << kUp);
  const float f = __uint_as_float((uint32_t)(127 - e) << 23);
  m = up;
  l *= f;
  return f * (1.f / (1 << kUp));
}

__global__ void __launch_bounds__(kThreads, kCtas)
paged8_attn_kernel(const __grid_constant__ CUtensorMap tmap, PagedSome p, const unsigned char* __restrict__ scale,
                   const __nv_bfloat16* __restrict__ q, __nv_bfloat16* __restrict__ out, float* __restrict__ lse,
                   int32_t* __restrict__ dev_status, Header* header, float* __restrict__ part, int part_rows, int max_parts,
                   int grp, float scale_log2) {
  extern __shared__ __align__(1024) unsigned char smem[];
  Shared& c = *reinterpret_cast<Shared*>(smem);
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, g8 = lane >> 2, t4 = lane & 3;
  const int tq = kRows / grp, H = p.G * grp, C = gridDim.x;
  if (tid < kCand) { c.plan.units[tid] = 0; c.plan.split[tid] = 0; c.plan.chunk[tid] = 0; }
  if (lane == 0) {
    for (int i = 0; i < kStages; ++i) mbar_init(&c.full[warp][i], 1);
    fence_mbar_init();
  }
  if (tid == 0) c.err = 0;
  __syncthreads();
  pdl_trigger();
  pdl_wait();
  const int open = blockIdx.x == 0 && tid == 0 ? header->open : 0;
  int longest, run = 1, units = 0, parts = 0;
  const float weight = plan_weight<kKeys>(p, tq, lane, longest);
  if (weight > 0.f) {                                               // (the same for the CTA) else every sequence is the other kernel's
    const int cand = plan_candidate(weight, longest, C, lane);
    plan_add<kKeys>(p, c.plan, tq, cand, warp, kWarps, lane);
    __syncthreads();
    plan_choose(c.plan, weight, cand, C, max_parts, kOverhead, lane, run, units, parts);
  }
  if (blockIdx.x == 0) {
    if (tid == 0) {
      if (open) raise_status(dev_status, VARRATE_ERR_CORRUPT);   // by a call whose merge did not run, or runs still
      header->run = run; header->units = units; header->parts = parts; header->open = 1;
    }
    for (int s = tid; s < p.S; s += kThreads) {
      SeqRange r;
      if (!seq_range(p, s, r)) raise_status(dev_status, VARRATE_ERR_CORRUPT);
    }
  }
  Walk<kKeys, PagedSome> w;
  if (warp == 0 && units > 0) w.load(p, tq, run, lane);
  int next = blockIdx.x;                                            // of warp 0
  uint32_t stage = 0, phase = 0;                                    // of the warp's next step
  bool ok = true;
  for (;;) {
    if (warp == 0) {
      SeqUnit x;
      int s = 0;
      x.valid = 0;
      while (next < units) {
        s = w.find(p, tq, tq, run, next, lane, x);
        int n = 0;
        if (lane == 0) n = take_unit(header, C, units);
        next = __shfl_sync(0xffffffffu, n, 0);
        if (x.t0 < x.t1) break;                                     // else: the block ends before this run
        x.valid = 0;
      }
      if (c.err) x.valid = 0;
      if (lane == 0) { x.seq = s; c.unit = x; }
    }
    __syncthreads();
    const SeqUnit x = c.unit;
    if (!x.valid) break;
    const int rows = x.ntok * grp, end = x.pos0 + x.ntok;
    // this warp's steps
    const int last = min(8 * x.t1, (end + 15) >> 4), st0 = 8 * x.t0 + warp, n = last > st0 ? (last - st0 + kWarps - 1) / kWarps : 0;
    Steps steps{p, scale, p.table + (int64_t)x.seq * p.max_pages, dev_status, x.g, st0, kWarps, n};
    steps.start(lane);
    const int to_v = p.G << p.page_log2;                            // rows from a key to its value
    auto request = [&](int i, uint32_t at) {                        // step i into stage `at`
      const int row = steps.row(steps.page(i), i);
      if (lane == 0) {
        mbar_arrive_expect_tx(&c.full[warp][at], kStepBytes);
        const uint32_t dst = smem_addr(c.ring[warp][at]);
        tma_load_2d(dst, &tmap, 0, row, &c.full[warp][at]);
        tma_load_2d(dst + kStepBytes / 2, &tmap, 0, row + to_v, &c.full[warp][at]);
      }
    };
    uint32_t ahead = stage;
    for (int i = 0; i < min(n, kStages); ++i) {
      request(i, ahead);
      ahead = ahead + 1 == kStages ? 0 : ahead + 1;
    }
    QueryFrags qf;
    const int gr = min(g8, rows - 1);                               // rows past the last one are it again, and not written
    qf.load(q + ((int64_t)(x.row0 + gr / grp) * H + x.g * grp + gr % grp) * kHeadDim, true, scale_log2, lane);
    const int sees0 = x.pos0 + min(2 * t4, rows - 1) / grp + 1, sees1 = x.pos0 + min(2 * t4 + 1, rows - 1) / grp + 1;   // keys that rows 2 t4, 2 t4 + 1 see
    float o[8][4];
#pragma unroll
    for (int j = 0; j < 8; ++j) o[j][0] = o[j][1] = o[j][2] = o[j][3] = 0.f;
    float m0 = 0.f, m1 = 0.f, l0 = 0.f, l1 = 0.f;                   // references, sums
    int unit = -1;                                                  // scale byte of the accumulator's unit, none yet

    int i = 0;
    for (; i < n; ++i) {
      ok = warp_wait(&c.full[warp][stage], phase);
      if (!ok) break;
      const unsigned char* tile = c.ring[warp][stage];
      const int key0 = (st0 + i * kWarps) << 4;
      const bool edge = key0 + 16 > x.pos0 + 1;                     // some row does not see all of its keys
      const uint32_t bytes = steps.bytes(i);
      const int bv = (int)(bytes >> 8);
      uint4 kq[4], vq[4];
      read_keys(tile, lane, kq);
      float sc[4];
      key_scores(kq, qf, sc);
      read_values(tile + kStepBytes / 2, lane, vq);
      // (of two extremes: no infinity that would make a number of a zero)
      const float f = __uint_as_float((bytes & 0xff) << 23), f0 = fminf(qf.f0 * f, FLT_MAX), f1 = fminf(qf.f1 * f, FLT_MAX);
      float x0 = sc[0] * f0, x1 = sc[1] * f1, x2 = sc[2] * f0, x3 = sc[3] * f1;
      if (edge) {
        const int a = key0 + g8, b = a + 8;
        if (a >= sees0) x0 = -INFINITY;
        if (a >= sees1) x1 = -INFINITY;
        if (b >= sees0) x2 = -INFINITY;
        if (b >= sees1) x3 = -INFINITY;
      }
      uint32_t nan[4];
      bool odd = false;
      if (edge) {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const int key = key0 + 2 * t4 + (i & 1) + 8 * (i >> 1);
          nan[i] = 0;
          if (key >= end) vq[i] = make_uint4(0, 0, 0, 0);
          else if (key > x.pos0) odd |= take_nan(vq[i], nan[i]);
        }
        odd = __any_sync(0xffffffffu, odd);
      }
      if (bv > unit) {                                              // (the same for the warp)
        if (unit >= 0) {
          const float down = exp2f((float)(unit - bv));
#pragma unroll
          for (int j = 0; j < 8; ++j) { o[j][0] *= down; o[j][1] *= down; o[j][2] *= down; o[j][3] *= down; }
        }
        unit = bv;
      }
      const float up = __uint_as_float((uint32_t)max(bv ? 127 + kUp + bv - unit : 127 + kUp, 0) << 23);
      const float low = bv ? __int_as_float(0x4b000000 + unit - bv) - (0x1p23f + kLow) : -kLow;   // (unit - bv >= 0 as a float, in two steps)
      // scores from the reference, and whether fp16 has its places for all of the step's weights (hidden ones are none)
      float y0, y1, y2, y3;
      auto fits = [&]() {
        y0 = x0 - m0; y1 = x1 - m1; y2 = x2 - m0; y3 = x3 - m1;
        float least = fminf(fminf(y0, y1), fminf(y2, y3));
        if (edge) least = fminf(fminf(y0 == -INFINITY ? 0.f : y0, y1 == -INFINITY ? 0.f : y1), fminf(y2 == -INFINITY ? 0.f : y2, y3 == -INFINITY ? 0.f : y3));
        return !__any_sync(0xffffffffu, fmaxf(fmaxf(y0, y1), fmaxf(y2, y3)) > kSlack || least < low);
      };
      bool direct = fits();
      if (!direct) {
        const float fa = move_reference(m0, l0, x0, x2, low), fb = move_reference(m1, l1, x1, x3, low);
        l0 *= fa;
        l1 *= fb;
#pragma unroll
        for (int j = 0; j < 8; ++j) { o[j][0] *= fa; o[j][2] *= fa; o[j][1] *= fb; o[j][3] *= fb; }
        direct = fits();
      }
      y0 = fast_exp2(y0); y1 = fast_exp2(y1); y2 = fast_exp2(y2); y3 = fast_exp2(y3);
      l0 += y0 + y2;
      l1 += y1 + y3;
      y0 *= up; y1 *= up; y2 *= up; y3 *= up;
      float z0 = y0, z1 = y1, z2 = y2, z3 = y3;
      if (!direct) {                                                // the others in bands of their own, below
        auto inside = [](float y) { return y >= kLeast && y <= kMost ? y : 0.f; };
        z0 = inside(y0); z1 = inside(y1); z2 = inside(y2); z3 = inside(y3);
        y0 -= z0; y1 -= z1; y2 -= z2; y3 -= z3;
      }
      uint32_t b0 = movmatrix_trans(pack_f16(z0, z1)), b1 = movmatrix_trans(pack_f16(z2, z3));
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        const uint32_t lo = value_bytes(vq[0], vq[1], j), hi = value_bytes(vq[2], vq[3], j);
        const uint32_t a[4] = {f16_codes(lo), f16_codes(lo >> 16), f16_codes(hi), f16_codes(hi >> 16)};
        mma_f16_16816(o[j], a, b0, b1);
      }
      if (!direct) {                                                // the largest weight of each band at 2^14
#pragma unroll 1
        for (int band = 0; band < kBands; ++band) {
          const uint32_t most = __reduce_max_sync(0xffffffffu, __float_as_uint(fmaxf(fmaxf(fmaxf(y0, y1), fmaxf(y2, y3)), 0.f)));
          if (most == 0) break;
          const float top = fmaxf(__uint_as_float(most), 0x1p-112f), to = __fdividef(0x1p14f, top), back = top * 0x1p-14f;
          auto inside = [&](float& y) { const float z = y * to; if (z >= kLeast) { y = 0.f; return z; } return 0.f; };
          z0 = inside(y0); z1 = inside(y1); z2 = inside(y2); z3 = inside(y3);
          b0 = movmatrix_trans(pack_f16(z0, z1)); b1 = movmatrix_trans(pack_f16(z2, z3));
#pragma unroll
          for (int j = 0; j < 8; ++j) {
            const uint32_t lo = value_bytes(vq[0], vq[1], j), hi = value_bytes(vq[2], vq[3], j);
            const uint32_t a[4] = {f16_codes(lo), f16_codes(lo >> 16), f16_codes(hi), f16_codes(hi >> 16)};
            float d[4] = {0.f, 0.f, 0.f, 0.f};
            mma_f16_16816(d, a, b0, b1);
#pragma unroll
            for (int i = 0; i < 4; ++i) o[j][i] = fmaf(d[i], back, o[j][i]);
          }
        }
      }
      if (odd) {                                                    // rare: NaN of keys that a part of the rows sees
#pragma unroll 1
        for (int k = 0; k < 16; ++k) {
          const int i = (k & 1) + 2 * (k >> 3), key = key0 + k;
          const uint32_t mine = i == 0 ? nan[0] : i == 1 ? nan[1] : i == 2 ? nan[2] : nan[3];
          const uint32_t bits = __shfl_sync(0xffffffffu, mine, (lane & ~3) | ((k & 7) >> 1));
#pragma unroll
          for (int j = 0; j < 8; ++j) {
            const bool a = bits >> (2 * j) & 1, b = bits >> (2 * j + 1) & 1;
            if (a && key < sees0) o[j][0] = NAN;
            if (a && key < sees1) o[j][1] = NAN;
            if (b && key < sees0) o[j][2] = NAN;
            if (b && key < sees1) o[j][3] = NAN;
          }
        }
      }
      __syncwarp();                                                 // the tile has been read
      if (i + kStages < n) request(i + kStages, stage);
      steps.done(i, lane);
      if (++stage == kStages) { stage = 0; phase ^= 1; }
    }
    if (!ok) {                                                      // no copy is in flight when the block ends
      for (int j = i; j < min(n, i + kStages); ++j) {
        warp_wait(&c.full[warp][stage], phase);
        if (++stage == kStages) { stage = 0; phase ^= 1; }
      }
      c.err = 1;
    }
    __syncthreads();                                                // the rings are empty
    // the warps' rows
#pragma unroll
    for (int i = 4; i < 32; i <<= 1) {
      l0 += __shfl_xor_sync(0xffffffffu, l0, i);
      l1 += __shfl_xor_sync(0xffffffffu, l1, i);
    }
    const float down0 = settle(m0, l0), down1 = settle(m1, l1);
    if (lane < 4) {
      c.m[warp][2 * lane] = m0; c.m[warp][2 * lane + 1] = m1;
      c.l[warp][2 * lane] = l0; c.l[warp][2 * lane + 1] = l1;
      if (lane == 0) c.u[warp] = max(unit, 0);
    }
    {                                                               // (a step that timed out leaves no part of its unit)
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        *reinterpret_cast<float2*>(&c.o[warp][2 * t4][16 * g8 + 2 * j]) = make_float2(o[j][0] * down0, o[j][2] * down0);
        *reinterpret_cast<float2*>(&c.o[warp][2 * t4 + 1][16 * g8 + 2 * j]) = make_float2(o[j][1] * down1, o[j][3] * down1);
      }
    }
    __syncthreads();
    if (warp < rows) {                                              // a row a warp, four elements a lane
      float mm = -INFINITY, ll = 0.f;
#pragma unroll
      for (int i = 0; i < kWarps; ++i) mm = fmaxf(mm, c.m[i][warp]);
      const float ref = mm == -INFINITY ? 0.f : mm;
#pragma unroll
      for (int i = 0; i < kWarps; ++i) ll += c.l[i][warp] * fast_exp2(c.m[i][warp] - ref);
      const float f = ll == 0.f ? 0.f : 1.f / ll;
      float4 y = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
      for (int i = 0; i < kWarps; ++i) {
        const float f1 = fast_exp2(c.m[i][warp] - ref) * f, f2 = __uint_as_float((uint32_t)c.u[i] << 23);   // normalised, then its unit
        const float4 v = *reinterpret_cast<const float4*>(&c.o[i][warp][4 * lane]);
        y.x += v.x * f1 * f2; y.y += v.y * f1 * f2; y.z += v.z * f1 * f2; y.w += v.w * f1 * f2;
      }
      const float at = ll == 0.f ? -INFINITY : ref + log2f(ll);
      if (x.slot < 0) {
        const int64_t i = (int64_t)(x.row0 + warp / grp) * H + x.g * grp + warp % grp;
        *reinterpret_cast<uint2*>(out + i * kHeadDim + 4 * lane) = make_uint2(pack_bf16(y.x, y.y), pack_bf16(y.z, y.w));
        if (lse && lane == 0) lse[i] = at * 0.69314718f;
      } else {
        const int64_t i = (int64_t)x.slot * part_rows + warp;
        *reinterpret_cast<float4*>(part + i * kHeadDim + 4 * lane) = y;
        if (lane == 0)
          reinterpret_cast<float2*>(part + (int64_t)max_parts * part_rows * kHeadDim)[i] = make_float2(at, ll == 0.f ? 0.f : 1.f);
      }
    }
    fence_proxy_async_smem();                                       // copies come where `o` was
    __syncthreads();
  }
  if (tid == 0 && c.err) {
    raise_status(dev_status, VARRATE_ERR_TIMEOUT);
    atomicExch(&header->gave_up, 1u);
  }
}

}  // namespace

size_t paged8_attn_ws_bytes(const Paged8& c, int group, int num_sms) {
  // The headers, both kernels' partials one after the other. By the rows alone, not by the sequences: a smaller batch never asks for
  // more, and may have chunks where a larger one of as many sequences as rows has none.
  const size_t mine = paged_part_bytes(c.p, group, kRows / group, num_sms);
  return c.p.T <= 2 * (8 / group) ? mine : mine + paged_part_bytes(c.p, group, 2 * (128 / group), num_sms) - kHeaderBytes;
}

int launch_paged8_attn(const Paged8& c, int layer, int group, const void* q, void* out, float* lse, int32_t* dev_status,
                       void* ws, int num_sms, cudaStream_t st) {
  const Paged& p = c.p;
  unsigned char* w = static_cast<unsigned char*>(ws);
  Header* header = reinterpret_cast<Header*>(w);
  float* part = reinterpret_cast<float*>(w + kHeaderBytes);
  const int tq = kRows / group, few = few_tokens(p, group);
  Merge8 two = {};
  two.lse = lse; two.few = few; two.tq2 = 128 / group;
  if (p.T > few) two.second = reinterpret_cast<float*>(w + paged_part_bytes(p, group, tq, num_sms));   // else no sequence can have more
  CUtensorMap tmap;
  if (!make_tmap_rows_u8(&tmap, p.pool + (int64_t)layer * p.layer_rows * kHeadDim, (uint64_t)p.layer_rows, 16)) return -1;
  static std::atomic<int> smem_set[64];
  int dev = 0;
  if (cudaGetDevice(&dev) != cudaSuccess || dev < 0 || dev >= 64 || smem_set[dev].load(std::memory_order_acquire) == 0) {
    if (cudaFuncSetAttribute(paged8_attn_kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)sizeof(Shared)) != cudaSuccess) return -1;
    if (dev >= 0 && dev < 64) smem_set[dev].store(1, std::memory_order_release);
  }
  auto many = [&]() { return launch_paged8_attn_tc(c, layer, group, few + 1, q, out, lse, dev_status, ws, two.second, num_sms, st); };
  if (!launch_pdl(paged8_attn_kernel, dim3(kCtas * num_sms), kThreads, sizeof(Shared), st, tmap, PagedSome{p, 0, few},
                  c.scale + (int64_t)layer * (p.layer_rows >> kBlockLog2),
                  (const __nv_bfloat16*)q, (__nv_bfloat16*)out, lse, dev_status, header, part, paged_part_rows(p, group, tq),
                  paged_max_parts(num_sms), group, kLog2e / sqrtf((float)kHeadDim)))
    return -1;
  if (two.second && many() < 0) return -1;
  return launch_paged8_merge(p, group, out, dev_status, ws, tq, two, num_sms, st) < 0 ? -1 : 2;
}

}  // namespace vr
