// Paged attention in 8 bits of sequences with many new tokens: tcgen05 products of codes that are widened on the way.
//
// The products, softmax, units and turns are those of the bf16 cache (paged_attn_tc.cu); what differs is how an operand comes
// to be. A row of K or V is 128 codes, a block of 16 rows has a scale 2^k. The tensor core's 8-bit products would take the
// codes as they are, but want the other side in 8 bits too, and weights or queries of 4 bits are no choice here. So four
// warps (kExpand; a row a thread) widen a tile where it lies: its codes land by TMA in the second half of its 32 KB, 128-byte
// swizzled, and are written over it as rows of 16 bits.
//   keys    to fp16, which holds every code, with no scale: one conversion for two codes. The scale of a block of 16 keys goes
//           into the factor that the softmax gives its scores anyway (key_scale), so that it costs nothing.
//   values  to bf16 times their scale: exact, a code has 4 bits and a scale none.
//   queries to fp16, a row times the power of two that brings its largest element into [2^14, 2^15) (row_to_f16): exact
//           but for elements below 2^-31 of it, which are off by 2^-39 of it at most; the factor is in the row's scale as well.
// Scores and outputs are sums of exact products in fp32, and weights are rounded to bf16 as for the bf16 cache.
//
// A row whose largest score is past 2^24 in size has its scores scaled down so that it is 2^24 (raise): then an ulp of it is 2 of log2
// units at most, not more than kRoom, and the weights stay below kMost. Where a later maximum is smaller in size (the scores before were
// far below 0) they are taken as they are again; references leave a unit as those of the scores themselves.
//
// Values come to be infinite only by a scale byte above 246, which append does not write; a code that is NaN counts as one
// where it is seen and as nothing elsewhere (warp 11, as in the bf16 kernel).
//
// Warps: 0-7 softmax, 8 producer, 9 and 10 issue, 11 values, 12-15 widen. Softmax threads have 184 registers, the others 72
// (setmaxnreg stands at the head of the two sides, or the compiler spills as if all had 128). Waits are bounded as in the
// bf16 kernel.
//
// Bound by the widening and the softmax side by side: 8192 tokens, 32 heads over 8, 441 us, 1250 TFLOP/s (0.65 of the
// measured bf16 rate; the bf16 cache, which has no widening, 336). Of the difference 40 us are the conversions (one instruction for
// two codes of a key; five for two of a value, which goes over fp32 to bf16 and meets its scale; without them, on zeros, it is 30 less), 25 the block of 512 threads, 20 the hop from the copy over the widening to the product, 20 the
// queries' scales and the block scales. A chunk of 383 tokens on 4000: 49.5 us with the kernel before and the merge, latency of the start (8 us before the
// first scores), three runs a block and partials of 252 rows.
// On the way, same prompt: keys to bf16 with their scale, and loops of the widening unrolled in full (the softmax's instructions
// are then fetched anew every tile), 528 us; registers not split, 1231 (spills). Without the
// turns that the two issuing warps take, 479.
#include <float.h>
#include <math.h>
#include <stddef.h>

#include <atomic>

#include <cudaTypedefs.h>

#include "common.cuh"
#include "decode_common.cuh"
#include "paged.h"
#include "paged8.h"
#include "paged8_tc.cuh"
#include "paged_plan.cuh"
#include "paged_tc.cuh"

namespace vr {

bool make_tmap_rows_u8(CUtensorMap* map, const void* base, uint64_t rows, uint32_t box_rows);
bool make_tmap_heads_bf16(CUtensorMap* map, const void* base, uint32_t heads, uint64_t rows, uint32_t box_heads, uint32_t box_rows);

namespace {

constexpr int kSoftWarps = 8, kProducer = 8, kIssuer = 9, kValues = 11;   // issuers: 9 and 10
constexpr int kExpand = 12, kExpandWarps = 4, kThreads = 32 * (kExpand + kExpandWarps);
// Registers a thread by warpgroup, softmax 0 and 1 and the others: 2 * 184 + 2 * 72 = 4 * 128 of the launch.
constexpr int kSoftRegs = 184, kOtherRegs = 72;
constexpr int kRows = 128, kKeys = kKeysBf16;
// As the plan counts them, in key tiles: a unit's start and output; the merge, with a partial's share. Against 2, 0 and 0: 23 chunks of 30 to 900
// tokens 162 us for 196, a prompt of 512 23.1 for 33.5 (not cut), other batches within 1 %; 3 to 6, 2 to 8 and 0 to 4 are as good.
constexpr float kOverhead = 4.f, kMerge = 4.f, kPart = 1.f;
constexpr int kTileBytes = kRows * kHeadDim * 2;            // a query, key or value tile
constexpr int kRing = 5;                                    // key and value tiles in flight, in turn
// The weights of a row sum to less than kMost, so that neither an accumulator nor the sum of the two warpgroups' overflows,
// whatever the values. kRoom (log2) is what scores may rise, and their number grow, before the reference moves: 8192 tokens,
// one key in 200 four times as long as the others, take 519 us at 24, 492 at 28, 468 at 32, 450 at 36, 441 at 40. What it costs is the low end: products with values below 2^-90 or so leave the range
// of fp32.
constexpr float kMost = 0.25f, kRoom = 40.f;

struct Ctl {
  uint64_t full[kRing], empty[kRing], look[kRing], looked[kRing];
  uint64_t s_full[2], p_half[2], p_full[2], o_half[2], o_full[2], q_full[2], q_seen[2], turn[2], drain[2];   // by warpgroup
  uint64_t raw[kRing], q_raw[2];                            // codes and bf16 queries, as they come
  uint64_t u_full[2], u_empty[2], u_looked[2], o1_full, o1_empty, planned;
  __align__(16) float key_scale[4][kKeys / kBlock];         // of the last key tiles' blocks
  SeqUnit unit[2];
  union {
    struct { float m[kRows], l[kRows]; int begun; } o1;                // second warpgroup's rows where both have one query tile
    PlanSums plan;
  };
  int16_t special[2][kHeadDim];                             // first position (from the first looked-at tile) of a NaN
  int any_special[2];
  int err;
  uint32_t tmem;
};
constexpr size_t kSmemBytes = 2 * kTileBytes + kRing * kTileBytes + sizeof(Ctl);
static_assert(kSmemBytes <= 232448, "shared memory of a block");

__global__ void __launch_bounds__(kThreads, 1)
paged8_attn_tc_kernel(const __grid_constant__ CUtensorMap tmap, const __grid_constant__ CUtensorMap tmap_q, PagedSome p,
                     const unsigned char* __restrict__ scale, __nv_bfloat16* __restrict__ out, float* __restrict__ lse,
                     int32_t* __restrict__ dev_status, Header* header,
                     float* __restrict__ part, int part_rows, int max_parts, int grp, float scale_log2) {
  extern __shared__ __align__(1024) unsigned char smem[];
  Ctl& c = *reinterpret_cast<Ctl*>(smem + (2 + kRing) * kTileBytes);
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const int tq = kRows / grp, bq = 2 * tq, H = p.G * grp, C = gridDim.x;
  const uint32_t q_addr = smem_addr(smem), ring = q_addr + 2 * kTileBytes;

  if (tid == 0) {
    for (int i = 0; i < kRing; ++i) {
      mbar_init(&c.raw[i], 1); mbar_init(&c.full[i], kExpandWarps); mbar_init(&c.empty[i], 2); mbar_init(&c.look[i], 1); mbar_init(&c.looked[i], 1);
    }
    for (int i = 0; i < 2; ++i) {
      mbar_init(&c.s_full[i], 1); mbar_init(&c.p_full[i], 4); mbar_init(&c.o_full[i], 1); mbar_init(&c.q_full[i], 4);
      mbar_init(&c.q_raw[i], 1);
      mbar_init(&c.q_seen[i], 1); mbar_init(&c.p_half[i], 4); mbar_init(&c.o_half[i], 1); mbar_init(&c.turn[i], 1);
      mbar_init(&c.drain[i], 1); mbar_init(&c.u_full[i], 1); mbar_init(&c.u_empty[i], kSoftWarps + 3 + kExpandWarps); mbar_init(&c.u_looked[i], 1);
    }
    mbar_init(&c.o1_full, 4); mbar_init(&c.o1_empty, 4); mbar_init(&c.planned, kThreads / 32);
    c.err = 0;
    fence_mbar_init();
  }
  if (tid < kCand) { c.plan.units[tid] = 0; c.plan.split[tid] = 0; c.plan.chunk[tid] = 0; }
  if (warp == kIssuer) tmem_alloc(&c.tmem, 512);
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tmem = c.tmem;
  pdl_trigger();
  pdl_wait();
  bool some = false;                                                // a sequence for this kernel, or it ends here
  for (int s = tid; s < p.S; s += kThreads) {
    SeqRange r;
    some |= plan_range(p, s, r) && r.n > 0;
  }
  if (!__syncthreads_or(some)) {
    if (blockIdx.x == 0 && tid == 0) {
      if (header->open) raise_status(dev_status, VARRATE_ERR_CORRUPT);
      header->run = 1; header->units = 0; header->parts = 0; header->open = 1;
    }
    if (warp == kIssuer) tmem_dealloc(tmem, 512);
    return;
  }
  // by a call whose merge did not run, or runs still
  const int open = blockIdx.x == 0 && warp == kProducer && lane == 0 ? header->open : 0;
  int longest;
  const float weight = plan_weight<kKeys>(p, bq, lane, longest);
  const int cand = plan_candidate(weight, longest, C, lane);
  plan_add<kKeys>(p, c.plan, bq, cand, warp, kThreads / 32, lane);
  __syncwarp();
  if (lane == 0) mbar_arrive(&c.planned);

  if (warp >= kSoftWarps) {
    fewer_registers<kOtherRegs>();
    if (warp == kProducer) {
      // ------------------------------------------------------------------ units, and their keys and values
      bool ok = wait_all(&c.planned, 0);
      int run = 1, units = 0, parts = 0;
      if (ok) plan_choose(c.plan, weight, cand, C, max_parts, kOverhead, lane, run, units, parts, kMerge, kPart);
      if (blockIdx.x == 0 && lane == 0) {
        if (open) raise_status(dev_status, VARRATE_ERR_CORRUPT);
        header->run = run; header->units = units; header->parts = parts; header->open = 1;
      }
      Walk<kKeys, PagedSome> w;
      w.load(p, bq, run, lane);
      const int page_keys = min(1 << p.page_log2, kKeys);           // rows of a box
      const int per_tile = kKeys / page_keys;
      int u = blockIdx.x;
      uint32_t n = 0;                                               // ring tiles so far
      for (uint32_t un = 0; ok; ++un) {
        SeqUnit x;
        int s = 0;
        x.valid = 0;
        while (u < units) {
          s = w.find(p, bq, tq, run, u, lane, x);
          if (x.t0 < x.t1) break;                                   // else: the block ends before this run
          x.valid = 0;
          if (lane == 0) u = take_unit(header, C, units);
          u = __shfl_sync(0xffffffffu, u, 0);
        }
        ok = wait_all(&c.u_empty[un & 1], ((un >> 1) & 1) ^ 1);
        if (!ok) break;
        if (lane == 0) {
          x.seq = s;
          c.unit[un & 1] = x;
          mbar_arrive(&c.u_full[un & 1]);
        }
        if (!x.valid) break;
        int next = 0;
        if (lane == 0) next = take_unit(header, C, units);
        const int32_t* table = p.table + (int64_t)s * p.max_pages;
        const int end = x.pos0 + x.ntok;
        auto page_at = [&](int t) {
          const int key = t * kKeys + lane * page_keys;
          return lane < per_tile && key < end ? __ldg(table + (key >> p.page_log2)) : 0;
        };
        int page = page_at(x.t0);
        for (int t = x.t0; t < x.t1 && ok; ++t) {
          const int key = t * kKeys + lane * page_keys;
          const bool mine = lane < per_tile && key < end;
          const int boxes = min(per_tile, (end - t * kKeys + page_keys - 1) / page_keys);
          int pg = page;
          if (mine && (pg < 0 || pg >= p.n_pages)) {
            raise_status(dev_status, VARRATE_ERR_CORRUPT);
            pg = 0;
          }
          const int row = (int)page_row(p, pg, 0, x.g, key & ((1 << p.page_log2) - 1));
          const int row_v = row + (p.G << p.page_log2);
          if (t + 1 < x.t1) page = page_at(t + 1);
#pragma unroll
          for (int kv = 0; kv < 2; ++kv, ++n) {
            const uint32_t slot = n % kRing;
            ok = ok && wait_all(&c.empty[slot], ((n / kRing) & 1) ^ 1);
            if (!ok) break;
            if (lane == 0) mbar_arrive_expect_tx(&c.raw[slot], (uint32_t)boxes * page_keys * 128);
            __syncwarp();
            if (mine)                                               // codes come to where the tile's second half will be
              tma_load_2d(ring + slot * kTileBytes + kKeys * 128 + lane * page_keys * 128, &tmap, 0, kv ? row_v : row, &c.raw[slot]);
            if (kv && t >= x.values_from && lane == 0) mbar_arrive(&c.look[slot]);
          }
        }
        u = __shfl_sync(0xffffffffu, next, 0);
      }
      if (!ok) {
        c.err = 1;
        const uint32_t oldest = n > kRing ? n - kRing : 0;          // no copy is in flight when the block ends
        for (uint32_t i = oldest; i < n; ++i) wait_all(&c.raw[i % kRing], (i / kRing) & 1);
      }
    } else if (warp == kIssuer || warp == kIssuer + 1) {
      // ------------------------------------------------------------------ products of warpgroup e
      // The warp stays together and its values are the same in every lane (broadcast from lane 0 where they come from
      // memory), so that descriptors stay in uniform registers; one elected lane issues. Both issuers pass every tile of
      // the ring in order, whether they use it or not.
      const int e = __shfl_sync(0xffffffffu, warp - kIssuer, 0);
      // queries and keys in fp16, weights and values in bf16
      constexpr uint32_t idesc_s = idesc_f16_f32(kRows, kKeys), idesc_o = idesc_bf16_f32(kRows, kHeadDim) | kBMn;
      const uint32_t tm = __shfl_sync(0xffffffffu, tmem, 0), ts = tm + 128 * e, to = tm + 256 + 128 * e;
      struct Ring { uint32_t slot, phase; };                        // a tile's place; two tiles further
      auto further = [](Ring& x) { x.slot += 2; if (x.slot >= kRing) { x.slot -= kRing; x.phase ^= 1; } };
      Ring key = {0, 0}, value = {1, 0};
      uint32_t looked = 0, par_p = 0, turns = e ^ 1;                // parities; the first warpgroup begins
      bool ok = true;
      for (uint32_t un = 0; ok; ++un) {
        ok = wait_all(&c.u_full[un & 1], (un >> 1) & 1);
        if (!ok) break;
        const Unit* x = &c.unit[un & 1];
        const int valid = __shfl_sync(0xffffffffu, x->valid, 0), t0 = __shfl_sync(0xffffffffu, x->t0, 0);
        const int nt = __shfl_sync(0xffffffffu, x->t1, 0) - t0, n_first = __shfl_sync(0xffffffffu, x->e0, 0) - t0;
        const int both = __shfl_sync(0xffffffffu, x->both, 0), from = __shfl_sync(0xffffffffu, x->values_from, 0) - t0;
        if (!valid) break;
        if (lane == 0) mbar_arrive(&c.u_empty[un & 1]);
        ok = wait_all(&c.q_full[e], un & 1);
        if (!ok) break;
        if (lane == 0) mbar_arrive(&c.q_seen[e]);
        auto mine = [&](int i) { return both ? (i & 1) == e : e || i < n_first; };
        auto scores = [&]() {                                       // issued by the elected lane
          const uint64_t a = sdesc_sw128(q_addr + e * kTileBytes), b = sdesc_sw128(ring + key.slot * kTileBytes);
#pragma unroll
          for (int ks = 0; ks < kHeadDim / 16; ++ks) {
            const uint64_t o = (uint64_t)((ks >> 2) * (kRows * 128) + (ks & 3) * 32) / 16;
            tc_mma_bf16(ts, a + o, b + o, idesc_s, ks != 0);
          }
          tc_commit(&c.s_full[e]);
          tc_commit(&c.empty[key.slot]);
        };
        auto pass = [&](Ring& x) {                                  // a tile that the other issuer uses alone
          if (!wait_all(&c.full[x.slot], x.phase)) return false;
          if (elect_one()) mbar_arrive(&c.empty[x.slot]);
          __syncwarp();
          further(x);
          return true;
        };
        auto next_scores = [&]() {                                  // by themselves, once the keys are there
          if (!wait_all(&c.full[key.slot], key.phase)) return false;
          tc_fence_after();
          if (elect_one()) scores();
          __syncwarp();
          further(key);
          return true;
        };
        // The keys of the first own tile; then per own tile its values, and the keys of the next one. Where both warpgroups
        // use a tile the products are queued behind one another, as a wait between them would hold them up; a decode step
        // waits for memory, and gives values back before it waits for keys.
        const int step = both ? 2 : 1;
        int ahead = 0;                                              // tiles whose keys are done
        for (; ok && ahead < nt && ahead < step && !mine(ahead); ++ahead) ok = pass(key);
        if (ok && ahead < nt && ahead < step) { ok = next_scores(); ++ahead; }
        uint32_t accumulate = 0;                                    // the accumulator holds products of this unit
        for (int i = 0; i < nt && ok; ++i) {
          const uint32_t slot = value.slot;
          if (!mine(i)) {
            if (!both && ahead == i) { ok = pass(key); ++ahead; }
            ok = ok && pass(value);
          } else {
            const bool queued = !both && ahead < nt && mine(ahead);
            ok = wait_all(&c.full[slot], value.phase);
            if (ok && i >= from) ok = wait_all(&c.looked[slot], (looked >> slot) & 1);
            if (ok && queued) ok = wait_all(&c.full[key.slot], key.phase);
            ok = ok && wait_all(&c.turn[e], turns & 1) && wait_all(&c.p_half[e], par_p);
            if (!ok) break;
            tc_fence_after();
            const uint64_t b = sdesc_sw128_mn(ring + slot * kTileBytes, kKeys * 128);
            if (elect_one()) {
#pragma unroll
              for (int ks = 0; ks < kKeys / 32; ++ks)
                tc_mma_bf16_ts(to, ts + 8 * ks, b + ks * (2048 / 16), idesc_o, ks ? 1 : accumulate);
              tc_commit(&c.o_half[e]);
            }
            __syncwarp();
            ok = wait_all(&c.p_full[e], par_p);
            if (!ok) break;
            par_p ^= 1;
            tc_fence_after();
            if (elect_one()) {
#pragma unroll
              for (int ks = kKeys / 32; ks < kKeys / 16; ++ks)
                tc_mma_bf16_ts(to, ts + 8 * ks, b + ks * (2048 / 16), idesc_o, 1);
              tc_commit(&c.o_full[e]);
              tc_commit(&c.empty[slot]);
              if (queued) scores();
              mbar_arrive(&c.turn[e ^ 1]);
            }
            __syncwarp();
            accumulate = 1;
            ++turns;
            further(value);
            if (queued) { further(key); ++ahead; }
            if (both) {
              for (; ok && ahead < nt && ahead < i + step; ++ahead) ok = pass(key);
              if (ok && ahead < nt) { ok = next_scores(); ++ahead; }
            }
          }
          if (i >= from) looked ^= 1u << slot;
        }
        // both issuers take as many turns in a unit
        const int all = both ? (nt + 1) / 2 : nt, own = both ? (nt + 1 - e) / 2 : e ? nt : min(n_first, nt);
        for (int i = own; i < all && ok; ++i, ++turns) {
          ok = wait_all(&c.turn[e], turns & 1);
          if (ok && elect_one()) mbar_arrive(&c.turn[e ^ 1]);
          __syncwarp();
        }
      }
      if (!ok) {                                                    // the products in flight end before TMEM is freed
        c.err = 1;
        if (elect_one()) tc_commit(&c.drain[e]);
        wait_all(&c.drain[e], 0);
      }
      __syncwarp();
    } else if (warp == kValues) {
      // ------------------------------------------------------------------ values that no row, or not every row, sees
      if (blockIdx.x == 0) {
        for (int s = lane; s < p.S; s += 32) {
          SeqRange r;
          if (!seq_range(p, s, r)) raise_status(dev_status, VARRATE_ERR_CORRUPT);
        }
      }
      // a lane looks at eight columns (chunk) of every second key
      const int panel = (lane >> 3) & 1, chunk = lane & 7, odd_key = lane >> 4;
      uint32_t n0 = 0, par = 0;
      bool ok = true;
      for (uint32_t un = 0; ok; ++un) {
        ok = wait_all(&c.u_full[un & 1], (un >> 1) & 1);
        if (!ok) break;
        const SeqUnit x = c.unit[un & 1];
        __syncwarp();
        if (!x.valid) break;
        int16_t first[8];
        bool any = false;
        const int end = x.pos0 + x.ntok;
        for (int t = x.values_from; t < x.t1; ++t) {
          const uint32_t n = n0 + 2 * (t - x.t0) + 1, slot = n % kRing;
          ok = wait_all(&c.look[slot], (par >> slot) & 1) && wait_all(&c.full[slot], (n / kRing) & 1);
          if (!ok) break;
          par ^= 1u << slot;
          const int lo = min(kKeys, max(0, x.pos0 + 1 - t * kKeys)), hi = min(kKeys, end - t * kKeys);
          unsigned char* v = smem + (2 + slot) * kTileBytes + panel * (kKeys * 128);
          auto at = [&](int key) { return reinterpret_cast<uint4*>(v + key * 128 + ((chunk ^ (key & 7)) << 4)); };
          // an exponent of all ones: infinity or NaN
          auto odd = [](uint32_t a) { return __vcmpeq2(a & 0x7f807f80u, 0x7f807f80u); };
          uint32_t found = 0;
#pragma unroll 4
          for (int key = lo + odd_key; key < hi; key += 2) {
            const uint4 w = *at(key);
            found |= odd(w.x) | odd(w.y) | odd(w.z) | odd(w.w);
          }
          if (__any_sync(0xffffffffu, found != 0)) {                // rare: element by element
            if (!any) {
#pragma unroll
              for (int i = 0; i < 8; ++i) first[i] = kNone;
            }
            any = true;
#pragma unroll 1
            for (int key = lo + odd_key; key < hi; key += 2) {
              const uint4 w = *at(key);
              uint32_t a[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
              for (int j = 0; j < 8; ++j) {
                const uint32_t h = (a[j >> 1] >> (16 * (j & 1))) & 0xffffu;
                if ((h & 0x7f80u) != 0x7f80u) continue;
                a[j >> 1] &= j & 1 ? 0x0000ffffu : 0xffff0000u;
                const int16_t pos = (int16_t)(t * kKeys + key - x.values_from * kKeys);
                first[j] = min(first[j], pos);
              }
              *at(key) = make_uint4(a[0], a[1], a[2], a[3]);
            }
            __syncwarp();
          }
#pragma unroll 4
          for (int key = hi + odd_key; key < kKeys; key += 2) *at(key) = make_uint4(0, 0, 0, 0);
          fence_proxy_async_smem();
          __syncwarp();
          if (lane == 0) mbar_arrive(&c.looked[slot]);
        }
        if (!ok) break;
        if (any) {                                                  // (the same in all lanes)
#pragma unroll
          for (int i = 0; i < 8; ++i) {
            const int other = __shfl_xor_sync(0xffffffffu, (int)first[i], 16);
            if (!odd_key) c.special[un & 1][64 * panel + 8 * chunk + i] = min(first[i], (int16_t)other);
          }
        }
        if (lane == 0) c.any_special[un & 1] = any;
        __syncwarp();
        if (lane == 0) {
          mbar_arrive(&c.u_looked[un & 1]);
          mbar_arrive(&c.u_empty[un & 1]);
        }
        n0 += 2 * (uint32_t)(x.t1 - x.t0);
      }
      if (!ok) c.err = 1;
    } else {
      // ------------------------------------------------------------------ codes to 16 bits: one key per thread
      const int key_in = tid - 32 * kExpand;
      uint32_t n = 0, n_k = 0;
      bool ok = true;
      for (uint32_t un = 0; ok; ++un) {
        ok = wait_all(&c.u_full[un & 1], (un >> 1) & 1);
        if (!ok) break;
        const SeqUnit& x = c.unit[un & 1];
        const int valid = x.valid, t0 = x.t0, t1 = x.t1, end = x.pos0 + x.ntok, g = x.g;
        const int32_t* table = p.table + (int64_t)x.seq * p.max_pages;
        __syncwarp();
        if (!valid) break;
        if (lane == 0) mbar_arrive(&c.u_empty[un & 1]);
        auto page_at = [&](int t) {
          const int key = t * kKeys + key_in;
          return t < t1 && key < end ? __ldg(table + (key >> p.page_log2)) : -1;
        };
        auto scales_at = [&](int t, int page, uint32_t& k, uint32_t& v) {   // (a page out of range: the producer raises the status)
          k = v = 0;
          if (page < 0 || page >= p.n_pages) return;
          const int64_t row = page_row(p, page, 0, g, (t * kKeys + key_in) & ((1 << p.page_log2) - 1));
          k = __ldg(scale + scale_at(row));
          v = __ldg(scale + scale_at(row + ((int64_t)p.G << p.page_log2)));
        };
        uint32_t sk, sv, sk1 = 0, sv1 = 0;
        scales_at(t0, page_at(t0), sk, sv);
        int page1 = page_at(t0 + 1);
        for (int t = t0; t < t1 && ok; ++t) {
          scales_at(t + 1, page1, sk1, sv1);
          page1 = page_at(t + 2);
          const bool there = t * kKeys + key_in < end;
#pragma unroll
          for (int kv = 0; kv < 2; ++kv, ++n) {
            const uint32_t slot = n % kRing;
            ok = ok && wait_all(&c.raw[slot], (n / kRing) & 1);
            if (!ok) break;
            if (kv) {
              expand_row<true>(smem + (2 + slot) * kTileBytes, kKeys, key_in, there, sv);
            } else {
              expand_row<false>(smem + (2 + slot) * kTileBytes, kKeys, key_in, there, 0);
              if ((key_in & (kBlock - 1)) == 0) c.key_scale[n_k & 3][key_in >> kBlockLog2] = __uint_as_float(sk << 23);
              ++n_k;
            }
            fence_proxy_async_smem();
            __syncwarp();
            if (lane == 0) mbar_arrive(&c.full[slot]);
          }
          sk = sk1;
          sv = sv1;
        }
      }
      if (!ok) c.err = 1;
    }
  } else {
    // ------------------------------------------------------------------ softmax: one row per thread
    more_registers<kSoftRegs>();
    const int e = warp >> 2, r = tid & 127, wrow = (warp & 3) * 32;
    const int tok_of = r / grp;                                   // of the query tile, and the row's place from its first one
    const int row_off = (tok_of * H + r % grp) * kHeadDim;
    const uint32_t lanes = (uint32_t)((warp & 3) * 32) << 16;
    const uint32_t ts = tmem + 128 * e + lanes, to = tmem + 256 + 128 * e + lanes;
    uint32_t n_k = 0;                                             // key tiles of the units before
    uint32_t n_s = 0, n_o = 0, n_both = 0, n_q = 0;               // score tiles, value products, merged units, query tiles so far
    bool ok = true;
    float ref = -INFINITY, l = 0.f;                               // reference, sum
    float down = 1.f;                                             // what a row's scores are multiplied by, and its reference is of
    bool unset = true;                                            // some row of the warp has no reference yet
    bool begun = false;                                           // the accumulator holds something of this unit
    // Pass nu: the queries of unit nu on their way, the output of unit nu - 1, the tiles of nu. (The code between the tiles
    // is kept short: it is fetched anew each time.)
    for (uint32_t nu = 0;; ++nu) {
      ok = wait_all(&c.u_full[nu & 1], (nu >> 1) & 1);
      if (!ok) break;
      const bool valid = c.unit[nu & 1].valid;
      // this warpgroup's query tile: the products that read the last one have ended, as its scores were all there; but where
      // the unit had no tile for this warpgroup, its copy may be on the way and the issuer may not have seen it
      n_q += valid;
      if (valid && wrow == 0 && nu > 0) {
        ok = wait_all(&c.q_seen[e], (nu - 1) & 1);
        if (!ok) break;
      }
      if (valid && wrow == 0 && lane == 0) {
        const SeqUnit& x = c.unit[nu & 1];
        mbar_arrive_expect_tx(&c.q_raw[e], (uint32_t)(tq * grp) * 256);
#pragma unroll
        for (int half = 0; half < 2; ++half)
          tma_load_3d(q_addr + e * kTileBytes + half * (kRows * 128), &tmap_q, half * 64, x.g * grp,
                      x.row0 + (x.both ? 0 : e * tq), &c.q_raw[e]);
      }
      __syncwarp();
      if (nu > 0) {
        const uint32_t un = nu - 1;
        const SeqUnit& x = c.unit[un & 1];
        const int tok0 = x.both ? 0 : e * tq, rows = min(tq, x.ntok - tok0) * grp;
        const bool live = wrow < rows, mine = r < rows;
        ok = wait_all(&c.u_looked[un & 1], (un >> 1) & 1);
        if (ok && begun) ok = wait_all(&c.o_full[e], (n_o - 1) & 1);
        if (!ok) break;
        tc_fence_after();
        if (l == 0.f) ref = -INFINITY;                              // nothing with a weight: no say in a merge
        if (down != 1.f) ref = (ref - kRoom) / down + kRoom;        // of the scores as they are, for lse and the merges
        float w0 = 1.f, w1 = 0.f;                                   // weights of the two warpgroups' values
        bool second = false;
        if (x.both) {
          if (e) {
            c.o1.m[r] = ref;
            c.o1.l[r] = l;
            if (r == 0) c.o1.begun = begun;
            tc_fence_before();
            __syncwarp();
            if (lane == 0) mbar_arrive(&c.o1_full);
            ok = wait_all(&c.o1_empty, n_both & 1);
            if (!ok) break;
          } else {
            ok = wait_all(&c.o1_full, n_both & 1);
            if (!ok) break;
            tc_fence_after();
            second = c.o1.begun;
            if (second) {
              const float m1 = c.o1.m[r], l1 = c.o1.l[r], mm = fmaxf(ref, m1), at = mm == -INFINITY ? 0.f : mm;
              w0 = fast_exp2(ref - at);
              w1 = fast_exp2(m1 - at);
              l = l * w0 + l1 * w1;
              ref = mm;
            }
          }
          ++n_both;
        }
        if (live && !(x.both && e)) {
          const int special = c.any_special[un & 1];
          const float f = l == 0.f ? 0.f : 1.f / l;
          const bool whole = x.slot < 0;                          // else a partial
          // 32 columns of the warp's rows at a time, 16-byte pieces exchanged between four lanes, so that a row's pieces leave
          // next to each other
          float* dst_part = part + ((int64_t)x.slot * part_rows + tok0 * grp + wrow) * kHeadDim;
          __nv_bfloat16* dst = out + ((int64_t)(x.row0 + tok0) * H + x.g * grp) * kHeadDim;
#pragma unroll 1
          for (int cb = 0; cb < kHeadDim; cb += 32) {
            float v[32];
            __syncwarp();
            if (begun) tmem_ld32(to + cb, v);
            if (second) {
              float v1[32];
              tmem_ld32(tmem + 384 + lanes + cb, v1);
#pragma unroll
              for (int k = 0; k < 32; ++k) v[k] = fmaf(v[k], w0, v1[k] * w1);
            }
            if (special) {
              const int at = x.pos0 + tok0 + tok_of + 1 - x.values_from * kKeys;   // positions below it are seen
              for (int k = 0; k < 32; ++k) {
                const int col = cb + k;
                if (c.special[un & 1][col] < at) add_at(v, k, NAN);
              }
            }
            if (whole) {
              uint4 y[4];
#pragma unroll
              for (int k = 0; k < 4; ++k)
                y[k] = make_uint4(pack_bf16(v[8 * k] * f, v[8 * k + 1] * f), pack_bf16(v[8 * k + 2] * f, v[8 * k + 3] * f),
                                  pack_bf16(v[8 * k + 4] * f, v[8 * k + 5] * f), pack_bf16(v[8 * k + 6] * f, v[8 * k + 7] * f));
              transpose4(y, lane);
#pragma unroll
              for (int i = 0; i < 4; ++i) {
                const int in = (lane & ~3) + i, off = __shfl_sync(0xffffffffu, row_off, in);
                if (wrow + in < rows) *reinterpret_cast<uint4*>(dst + off + cb + 8 * (lane & 3)) = y[i];
              }
            } else if (begun) {
#pragma unroll
              for (int h = 0; h < 2; ++h) {
                uint4 y[4];
#pragma unroll
                for (int k = 0; k < 4; ++k)
                  y[k] = make_uint4(__float_as_uint(v[16 * h + 4 * k]), __float_as_uint(v[16 * h + 4 * k + 1]),
                                    __float_as_uint(v[16 * h + 4 * k + 2]), __float_as_uint(v[16 * h + 4 * k + 3]));
                transpose4(y, lane);
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                  const int in = (lane & ~3) + i;
                  if (wrow + in < rows)
                    *reinterpret_cast<uint4*>(dst_part + (int64_t)in * kHeadDim + cb + 16 * h + 4 * (lane & 3)) = y[i];
                }
              }
            }
          }
          if (mine && whole && lse)
            lse[(int64_t)(x.row0 + tok0 + tok_of) * H + x.g * grp + r % grp] = l == 0.f ? -INFINITY : (ref + log2f(l)) * 0.69314718f;
          if (mine && !whole && begun) {
            float* ml = part + (int64_t)max_parts * part_rows * kHeadDim;
            *reinterpret_cast<float2*>(ml + ((int64_t)x.slot * part_rows + tok0 * grp + r) * 2) = make_float2(ref, l);
          }
          tc_fence_before();
        }
        if (x.both && !e) {
          __syncwarp();
          if (lane == 0) mbar_arrive(&c.o1_empty);
        }
        __syncwarp();
        if (lane == 0) mbar_arrive(&c.u_empty[un & 1]);
      }
      if (!valid) break;
      const SeqUnit& x = c.unit[nu & 1];
      const int both = x.both, tok0 = both ? 0 : e * tq, rows = min(tq, x.ntok - tok0) * grp;
      const bool live = wrow < rows, mine = r < rows;
      const int sees = x.pos0 + tok0 + tok_of + 1;                // keys that this row sees
      const int first_sees = __shfl_sync(0xffffffffu, sees, 0);   // the least of the warp
      const int step = both ? 2 : 1, last = both || e ? x.t1 : x.e0;
      const int t_first = x.t0, tiles = x.t1 - x.t0;
      ref = -INFINITY;
      l = 0.f;
      down = 1.f;
      unset = true;
      begun = false;
      float row_scale = scale_log2;
      // the queries in fp16, and what that takes off their size
      ok = wait_all(&c.q_raw[e], (n_q - 1) & 1);
      if (!ok) break;
      row_scale *= row_to_f16(smem + e * kTileBytes, kRows, r);
      fence_proxy_async_smem();
      __syncwarp();
      if (lane == 0) mbar_arrive(&c.q_full[e]);
      for (int t = x.t0 + (both ? e : 0); t < last; t += step) {
        ok = wait_all(&c.s_full[e], n_s & 1);
        if (!ok) break;
        ++n_s;
        tc_fence_after();
        if (live) {
          const int lim = sees - t * kKeys;
          const bool cut = first_sees - t * kKeys < kKeys;        // some row of the warp does not see the whole tile
          auto hide = [&](int cb, float (&s)[32]) {
            if (cut) {
#pragma unroll
              for (int k = 0; k < 32; ++k) s[k] = cb + k < lim ? s[k] : -INFINITY;
            }
          };
          // The weights from the reference as it is, in halves of 64 keys, each handed on by itself. If the row's sum is no
          // number below kMost with them: the maximum of the scores first, then the weights again.
          float x[32];
          uint32_t pk[32];
          // what a score of a block of keys is multiplied by (neither an infinity, for scores of 0, nor 0, for hidden ones)
          auto block_scale = [&](int b) {
            return fminf(fmaxf(row_scale * c.key_scale[(n_k + (t - t_first)) & 3][b], FLT_MIN), FLT_MAX);
          };
          auto block_scales = [&](int b, float (&y)[4]) {
            const float4 k = *reinterpret_cast<const float4*>(&c.key_scale[(n_k + (t - t_first)) & 3][b]);
            const float z[4] = {k.x, k.y, k.z, k.w};
#pragma unroll
            for (int i = 0; i < 4; ++i) y[i] = fminf(fmaxf(row_scale * z[i], FLT_MIN), FLT_MAX);
          };
          auto weights = [&](int cb0) {
            const float off1 = ref == -INFINITY ? 0.f : -ref;
            const float2 off = make_float2(off1, off1);
            float sc1[4];                                           // by 16 keys
            block_scales(cb0 / kBlock, sc1);
            float2 sum[2] = {make_float2(0.f, 0.f), make_float2(0.f, 0.f)};
            float s[64];
            tmem_ld64(ts + cb0, s);
            if (cut) {
#pragma unroll
              for (int k = 0; k < 64; ++k) s[k] = cb0 + k < lim ? s[k] : -INFINITY;
            }
#pragma unroll
            for (int k = 0; k < 32; ++k) {
              const float2 a = fma2(make_float2(s[2 * k], s[2 * k + 1]), make_float2(sc1[k / 8], sc1[k / 8]), off);
              s[2 * k] = fast_exp2(a.x);
              s[2 * k + 1] = fast_exp2(a.y);
            }
#pragma unroll
            for (int k = 0; k < 32; ++k) {
              const float2 w = make_float2(s[2 * k], s[2 * k + 1]);
              sum[k & 1] = add2(sum[k & 1], w);
              pk[k] = pack_bf16(w.x, w.y);
            }
            sum[0] = add2(sum[0], sum[1]);
            return sum[0].x + sum[0].y;
          };
          // the reference up to kRoom above the maximum of the scores from column cb on; `some`: up to the first 32 that show one
          auto raise = [&](int cb, bool some) {
            float mx = -INFINITY;
#pragma unroll 1
            for (bool first = true; cb < kKeys && (first || !some || __any_sync(0xffffffffu, mine && mx == -INFINITY)); cb += 32, first = false) {
              tmem_ld32(ts + cb, x);
              hide(cb, x);
              const float b0 = block_scale(cb / kBlock), b1 = block_scale(cb / kBlock + 1);
#pragma unroll
              for (int k = 0; k < 32; ++k) x[k] *= k < 16 ? b0 : b1;
              float top[4] = {mx, x[0], x[1], x[2]};
#pragma unroll
              for (int k = 3; k < 32; ++k) top[k & 3] = fmaxf(top[k & 3], x[k]);
              mx = fmaxf(fmaxf(top[0], top[1]), fmaxf(top[2], top[3]));
            }
            const float up = (l < 0.5f * kMost ? mx : fmaxf(mx, ref)) + kRoom;   // a sum that has grown makes room too
            float f = 1.f;
            if (mine && up > ref) {
              f = ref == -INFINITY ? 0.f : fast_exp2(ref - up);
              ref = up;
              // So large that a rounding of the reference is not small beside kRoom: the row's scores are taken at 2^24 from here on,
              // as long as the maximum is of that size. They are not known to a unit, the largest decides alone, and does so as well
              // where they are smaller.
              const float whole = mx / down, size = fabsf(whole);   // (exact: a power of two)
              const float to = size > 0x1p24f ? __uint_as_float((uint32_t)(127 + 127 + 23 - (int)(__float_as_uint(size) >> 23)) << 23) : 1.f;
              if (up == mx + kRoom && size < INFINITY && to != down) {
                row_scale *= to / down;
                down = to;
                ref = fmaf(whole, to, kRoom);
              }
            }
            return f;
          };
          auto rescale = [&](float f) {                           // the accumulator, whose products have ended
            tc_fence_after();
#pragma unroll 1
            for (int cb = 0; cb < kHeadDim; cb += 32) {
              tmem_ld32(to + cb, x);
#pragma unroll
              for (int k = 0; k < 32; ++k) x[k] *= f;
              tmem_st32(to + cb, x);
            }
          };
          // (fminf: where l is no number already the weights are as good as any)
          auto unusable = [&](float sum) { return __any_sync(0xffffffffu, mine && !(sum < fminf(kMost - l, kMost))); };
          // one body for both halves: the loop has to be short, instructions are fetched anew when it is not
#pragma unroll 1
          for (int half = 0; half < 2; ++half) {
            float total;
            bool tried = false;
            for (;;) {
              if (tried || (unset && half == 0)) {                // (the same for the warp)
                const float f = raise(64 * half, !tried);
                l *= f;
                if (begun || half) {                              // the accumulator's last products have ended
                  ok = wait_all(half ? &c.o_half[e] : &c.o_full[e], half ? n_o & 1 : (n_o - 1) & 1);
                  if (!ok) break;
                  rescale(f);
                }
              }
              total = weights(64 * half);
              if (tried || !unusable(total)) break;
              tried = true;
            }
            if (!ok) break;
            tmem_st32(ts + 32 * half, reinterpret_cast<const float(&)[32]>(pk));   // in place of the scores
            l += total;
            tmem_wait_st();
            tc_fence_before();
            __syncwarp();
            if (lane == 0) mbar_arrive(half ? &c.p_full[e] : &c.p_half[e]);
          }
          if (!ok) break;
        } else if (lane == 0) {
          mbar_arrive(&c.p_half[e]);
          mbar_arrive(&c.p_full[e]);
        }
        begun = true;
        ++n_o;
        unset = __any_sync(0xffffffffu, mine && ref == -INFINITY);
      }
      if (!ok) break;
      n_k += tiles;
    }
    if (!ok) {
      c.err = 1;
      if (n_q > 0) wait_all(&c.q_raw[e], (n_q - 1) & 1);   // no copy is in flight when the block ends
    }
  }
  __syncthreads();
  if (warp == kIssuer) tmem_dealloc(tmem, 512);
  if (tid == 0 && c.err) {
    raise_status(dev_status, VARRATE_ERR_TIMEOUT);
    atomicExch(&header->gave_up, 1u);
  }
}

}  // namespace

int launch_paged8_attn_tc(const Paged8& c, int layer, int group, int n_min, const void* q, void* out, float* lse,
                          int32_t* dev_status, void* ws, float* part, int num_sms, cudaStream_t st) {
  const PagedSome p{c.p, n_min, INT32_MAX};
  static std::atomic<int> smem_set[64];
  int dev = 0;
  if (cudaGetDevice(&dev) != cudaSuccess || dev < 0 || dev >= 64 || smem_set[dev].load(std::memory_order_acquire) == 0) {
    if (!registers_for(paged8_attn_tc_kernel, kThreads, 128 * (2 * kSoftRegs + 2 * kOtherRegs))) return -1;
    if (cudaFuncSetAttribute(paged8_attn_tc_kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)kSmemBytes) != cudaSuccess) return -1;
    if (dev >= 0 && dev < 64) smem_set[dev].store(1, std::memory_order_release);
  }
  CUtensorMap tmap, tmap_q;
  const int ps = 1 << p.page_log2, tq = kRows / group;
  if (!make_tmap_rows_u8(&tmap, p.pool + (int64_t)layer * p.layer_rows * kHeadDim, (uint64_t)p.layer_rows, ps < kKeys ? ps : kKeys)) return -1;
  if (!make_tmap_heads_bf16(&tmap_q, q, (uint32_t)(p.G * group), (uint64_t)p.T, (uint32_t)group, (uint32_t)tq)) return -1;
  return launch_pdl(paged8_attn_tc_kernel, dim3(num_sms), kThreads, kSmemBytes, st, tmap, tmap_q, p,
                    c.scale + (int64_t)layer * (p.layer_rows >> kBlockLog2), (__nv_bfloat16*)out, lse, dev_status,
                    reinterpret_cast<Header*>(static_cast<unsigned char*>(ws) + kSecondHeader), part, paged_part_rows(p, group, 2 * tq),
                    paged_max_parts(num_sms), group, kLog2e / sqrtf((float)kHeadDim))
             ? 1 : -1;
}

}  // namespace vr
