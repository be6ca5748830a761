// Paged cache, attention of new tokens, bf16: tcgen05 products fed by TMA out of the pages.
//
// The rows of a query tile are (token, query head) pairs of one KV head, at most 128: tq = 128 / group tokens. Per tile
// of 128 keys
//   scores  S[row][key] = Q[row][.] K[key][.]     M = 128, N = 128, K = 128, both operands in shared memory
//   values  O[row][.]  += P[row][key] V[key][.]   M = 128, N = 128, K = keys, P (bf16) from TMEM over the scores
// A page holds a head's keys (and values) as rows of 256 bytes, so a tile is one TMA box of 64 columns per page and half
// row; 128-byte swizzle; keys are the K-major B operand, values the MN-major one.
// Two softmax warpgroups (thread = row) work in turn, so that the products of one run under the softmax of the other:
//   a block of more than tq new tokens gives each warpgroup a query tile of its own, and both use every key tile;
//   a smaller one (a decode step) gives both the same query tile and every second key tile, merged at the end.
// The reference of a row (log2 units) stands kRoom above the maximum of its first 32 scores and moves only when its weights would
// sum to kMost: then to kRoom above the maximum, and its accumulator is rescaled in TMEM. So a tile is read once, without a
// maximum, and as the weights sum to less than 1, accumulators stay below the largest value.
// Weights are handed on in halves of 64 keys: the products of the first run while the second is made.
//
// Units of work (paged_plan.cuh) are taken by one CTA per SM: the first by its number, the others from a counter in the
// workspace; paged_attn_merge_kernel merges the partials.
//
// Values at positions that a row does not see have weight 0 in P, and 0 times an infinity is no number: in the tiles
// where that can happen one warp zeroes every value past the block's last token, and values that are not finite and
// that only a part of the block's tokens sees are zeroed too, remembered (Ctl::special) and added to the rows that see them.
//
// Warps: 0-3, 4-7 softmax; 8 TMA producer of keys and values; 9, 10 issue the products of one softmax warpgroup each (the
// tensor core takes few products ahead, so that a single issuing warp's waits would stand in its way), in turns of a tile,
// which keeps the warpgroups half a period apart; 11 values. Every wait is bounded; one that gives up raises
// VARRATE_ERR_TIMEOUT, its CTA takes no further unit and ends after its copies and products in flight have.
//
// Bound by the tensor cores for prompts: 8192 tokens, 32 heads over 8: 335 us, 1640 TFLOP/s (88 % of the rate of a large bf16
// product) in captured runs of 24 calls, 361 us, 1520 as calls one after another for longer, where the power limit shows; 512 tokens on
// 131072: 653 us, 1680 (90 %), and 709 us. By memory for decode steps: eight sequences of 32768 tokens
// 171 us, 6.3 TB/s (93 % of a copy). By latency for short ones: 900 tokens of one sequence 14.3 us, two launches and
// one pass through code that is not in the instruction caches; a unit costs 2 to 4 us beside its tiles (output, queries, first scores).
// What was measured on the way, on that prompt, captured: one issuing warp 609 us, its values in uniform registers 569, two issuing
// warps 541, in turns and with the weights in halves 474, no maximum in the steady state 427, output and
// queries in short coalesced loops 405, one threshold for the reference and no votes ahead of the weights 369, one body for
// both halves with 64 scores a load 342, queries by TMA 333. With a maximum of every tile 473 instead of 427, without the
// turns 448; with the output in a function that is not inlined 406 instead of 366. The bound on
// the sum of a row's weights costs 1 %. Partials merged by the last CTA of a block instead of a kernel: 89 to 117 us instead of 76 on a mixed
// step, whose partials are 252 rows, as its loads stand in the way of the next unit; not measured where every block is one token.
#include <math.h>
#include <stddef.h>

#include <atomic>

#include <cudaTypedefs.h>

#include "common.cuh"
#include "decode_common.cuh"
#include "paged.h"
#include "paged_plan.cuh"
#include "paged_tc.cuh"

namespace vr {

bool make_tmap_rows_bf16(CUtensorMap* map, const void* base, uint64_t rows, uint32_t box_rows);
bool make_tmap_heads_bf16(CUtensorMap* map, const void* base, uint32_t heads, uint64_t rows, uint32_t box_heads, uint32_t box_rows);

namespace {

constexpr int kThreads = 384;
constexpr int kSoftWarps = 8, kProducer = 8, kIssuer = 9, kValues = 11;   // issuers: 9 and 10
constexpr int kRows = 128, kKeys = kKeysBf16;
constexpr float kOverhead = 2.f;                            // of a unit, in key tiles, as the plan counts it: geometric mean over
                                                            // 19 cases 42.0 us, at 3 and 4 41.8, at 6 42.1, at 8 42.5
constexpr int kTileBytes = kRows * kHeadDim * 2;            // a query, key or value tile
constexpr int kRing = 5;                                    // key and value tiles in flight, in turn
// The weights of a row sum to less than kMost, so that neither an accumulator nor the sum of the two warpgroups' overflows,
// whatever the values. kRoom (log2) is what scores may rise, and their number grow, before the reference moves: 8192 tokens,
// one key in 200 four times as long as the others, take 411 us at 24, 392 at 28, 377 at 32, 366 at 36, 361 at 40 (357 with no bound on
// the sum of a row, 2^40 for half a tile's). What it costs is the low end: products with values below 2^-90 or so leave the range
// of fp32.
constexpr float kMost = 0.25f, kRoom = 40.f;

struct Ctl {
  uint64_t full[kRing], empty[kRing], look[kRing], looked[kRing];
  uint64_t s_full[2], p_half[2], p_full[2], o_half[2], o_full[2], q_full[2], q_seen[2], turn[2], drain[2];   // by warpgroup
  uint64_t u_full[2], u_empty[2], u_looked[2], o1_full, o1_empty, planned;
  Unit unit[2];
  union {
    struct { float m[kRows], l[kRows]; int begun; } o1;                // second warpgroup's rows where both have one query tile
    PlanSums plan;
  };
  int16_t special[2][3][kHeadDim];                          // first position (from the first looked-at tile) of +inf, -inf, NaN
  int any_special[2];
  int err;
  uint32_t tmem;
};
constexpr size_t kSmemBytes = 2 * kTileBytes + kRing * kTileBytes + sizeof(Ctl);
static_assert(kSmemBytes <= 232448, "shared memory of a block");

__global__ void __launch_bounds__(kThreads, 1)
paged_attn_tc_kernel(const __grid_constant__ CUtensorMap tmap, const __grid_constant__ CUtensorMap tmap_q, Paged p,
                     __nv_bfloat16* __restrict__ out, int32_t* __restrict__ dev_status, Header* header,
                     float* __restrict__ part, int part_rows, int max_parts, int grp, float scale_log2) {
  extern __shared__ __align__(1024) unsigned char smem[];
  Ctl& c = *reinterpret_cast<Ctl*>(smem + (2 + kRing) * kTileBytes);
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const int tq = kRows / grp, bq = 2 * tq, H = p.G * grp, C = gridDim.x;
  const uint32_t q_addr = smem_addr(smem), ring = q_addr + 2 * kTileBytes;

  pdl_trigger();
  if (tid == 0) {
    for (int i = 0; i < kRing; ++i) {
      mbar_init(&c.full[i], 1); mbar_init(&c.empty[i], 2); mbar_init(&c.look[i], 1); mbar_init(&c.looked[i], 1);
    }
    for (int i = 0; i < 2; ++i) {
      mbar_init(&c.s_full[i], 1); mbar_init(&c.p_full[i], 4); mbar_init(&c.o_full[i], 1); mbar_init(&c.q_full[i], 1);
      mbar_init(&c.q_seen[i], 1); mbar_init(&c.p_half[i], 4); mbar_init(&c.o_half[i], 1); mbar_init(&c.turn[i], 1);
      mbar_init(&c.drain[i], 1); mbar_init(&c.u_full[i], 1); mbar_init(&c.u_empty[i], kSoftWarps + 3); mbar_init(&c.u_looked[i], 1);
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
  pdl_wait();
  // by a call whose merge did not run, or runs still
  const int open = blockIdx.x == 0 && warp == kProducer && lane == 0 ? header->open : 0;
  int longest;
  const float weight = plan_weight<kKeys>(p, bq, lane, longest);
  const int cand = plan_candidate(weight, longest, C, lane);
  plan_add<kKeys>(p, c.plan, bq, cand, warp, kThreads / 32, lane);
  __syncwarp();
  if (lane == 0) mbar_arrive(&c.planned);

  if (warp == kProducer) {
    // ------------------------------------------------------------------ units, and their keys and values
    bool ok = wait_all(&c.planned, 0);
    int run = 1, units = 0, parts = 0;
    if (ok) plan_choose(c.plan, weight, cand, C, max_parts, kOverhead, lane, run, units, parts);
    if (blockIdx.x == 0 && lane == 0) {
      if (open) raise_status(dev_status, VARRATE_ERR_CORRUPT);
      header->run = run; header->units = units; header->parts = parts; header->open = 1;
    }
    Walk<kKeys> w;
    w.load(p, bq, run, lane);
    const int page_keys = min(1 << p.page_log2, kKeys);           // rows of a box
    const int per_tile = kKeys / page_keys;
    int u = blockIdx.x;
    uint32_t n = 0;                                               // ring tiles so far
    for (uint32_t un = 0; ok; ++un) {
      Unit x;
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
        c.unit[un & 1] = x;
        mbar_arrive(&c.u_full[un & 1]);
      }
      if (!x.valid) break;
      int next = 0;
      if (lane == 0) next = take_unit(header, C, units);
      const int32_t* table = p.table + (int64_t)s * p.max_pages;
      const int end = x.pos0 + x.ntok;
      const int piece = lane >> 1, half = lane & 1;               // this lane's box of a tile
      auto page_at = [&](int t) {
        const int key = t * kKeys + piece * page_keys;
        return piece < per_tile && key < end ? __ldg(table + (key >> p.page_log2)) : 0;
      };
      int page = page_at(x.t0);
      for (int t = x.t0; t < x.t1 && ok; ++t) {
        const int key = t * kKeys + piece * page_keys;
        const bool mine = piece < per_tile && key < end;
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
          if (lane == 0) mbar_arrive_expect_tx(&c.full[slot], (uint32_t)boxes * page_keys * 256);
          __syncwarp();
          if (mine)
            tma_load_2d(ring + slot * kTileBytes + half * (kKeys * 128) + piece * page_keys * 128, &tmap, half * 64,
                        kv ? row_v : row, &c.full[slot]);
          if (kv && t >= x.values_from && lane == 0) mbar_arrive(&c.look[slot]);
        }
      }
      u = __shfl_sync(0xffffffffu, next, 0);
    }
    if (!ok) {
      c.err = 1;
      const uint32_t oldest = n > kRing ? n - kRing : 0;          // no copy is in flight when the block ends
      for (uint32_t i = oldest; i < n; ++i) wait_all(&c.full[i % kRing], (i / kRing) & 1);
    }
  } else if (warp == kIssuer || warp == kIssuer + 1) {
    // ------------------------------------------------------------------ products of warpgroup e
    // The warp stays together and its values are the same in every lane (broadcast from lane 0 where they come from
    // memory), so that descriptors stay in uniform registers; one elected lane issues. Both issuers pass every tile of
    // the ring in order, whether they use it or not.
    const int e = __shfl_sync(0xffffffffu, warp - kIssuer, 0);
    constexpr uint32_t idesc_s = idesc_bf16_f32(kRows, kKeys), idesc_o = idesc_bf16_f32(kRows, kHeadDim) | kBMn;
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
      const Unit x = c.unit[un & 1];
      __syncwarp();
      if (!x.valid) break;
      int16_t first[8][3];
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
            for (int i = 0; i < 24; ++i) first[i / 3][i % 3] = kNone;
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
              if (h & 0x7f) first[j][2] = min(first[j][2], pos);
              else if (h >> 15) first[j][1] = min(first[j][1], pos);
              else first[j][0] = min(first[j][0], pos);
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
        for (int i = 0; i < 24; ++i) {
          const int other = __shfl_xor_sync(0xffffffffu, (int)first[i / 3][i % 3], 16);
          if (!odd_key) c.special[un & 1][i % 3][64 * panel + 8 * chunk + i / 3] = min(first[i / 3][i % 3], (int16_t)other);
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
    // ------------------------------------------------------------------ softmax: one row per thread
    const int e = warp >> 2, r = tid & 127, wrow = (warp & 3) * 32;
    const int tok_of = r / grp;                                   // of the query tile, and the row's place from its first one
    const int row_off = (tok_of * H + r % grp) * kHeadDim;
    const uint32_t lanes = (uint32_t)((warp & 3) * 32) << 16;
    const uint32_t ts = tmem + 128 * e + lanes, to = tmem + 256 + 128 * e + lanes;
    uint32_t n_s = 0, n_o = 0, n_both = 0, n_q = 0;               // score tiles, value products, merged units, query tiles so far
    bool ok = true;
    float ref = -INFINITY, l = 0.f;                               // reference, sum
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
        const Unit& x = c.unit[nu & 1];
        mbar_arrive_expect_tx(&c.q_full[e], (uint32_t)(tq * grp) * 256);
#pragma unroll
        for (int half = 0; half < 2; ++half)
          tma_load_3d(q_addr + e * kTileBytes + half * (kRows * 128), &tmap_q, half * 64, x.g * grp,
                      x.row0 + (x.both ? 0 : e * tq), &c.q_full[e]);
      }
      __syncwarp();
      if (nu > 0) {
        const uint32_t un = nu - 1;
        const Unit& x = c.unit[un & 1];
        const int tok0 = x.both ? 0 : e * tq, rows = min(tq, x.ntok - tok0) * grp;
        const bool live = wrow < rows, mine = r < rows;
        ok = wait_all(&c.u_looked[un & 1], (un >> 1) & 1);
        if (ok && begun) ok = wait_all(&c.o_full[e], (n_o - 1) & 1);
        if (!ok) break;
        tc_fence_after();
        if (l == 0.f) ref = -INFINITY;                              // nothing with a weight: no say in a merge
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
                float y = 0.f;
                if (c.special[un & 1][0][col] < at) y += INFINITY;
                if (c.special[un & 1][1][col] < at) y -= INFINITY;
                if (c.special[un & 1][2][col] < at) y = NAN;
                add_at(v, k, y);
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
      const Unit& x = c.unit[nu & 1];
      const int both = x.both, tok0 = both ? 0 : e * tq, rows = min(tq, x.ntok - tok0) * grp;
      const bool live = wrow < rows, mine = r < rows;
      const int sees = x.pos0 + tok0 + tok_of + 1;                // keys that this row sees
      const int first_sees = __shfl_sync(0xffffffffu, sees, 0);   // the least of the warp
      const int step = both ? 2 : 1, last = both || e ? x.t1 : x.e0;
      ref = -INFINITY;
      l = 0.f;
      unset = true;
      begun = false;
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
          auto weights = [&](int cb0) {
            const float off1 = ref == -INFINITY ? 0.f : -ref;
            const float2 sc = make_float2(scale_log2, scale_log2), off = make_float2(off1, off1);
            float2 sum[2] = {make_float2(0.f, 0.f), make_float2(0.f, 0.f)};
            float s[64];
            tmem_ld64(ts + cb0, s);
            if (cut) {
#pragma unroll
              for (int k = 0; k < 64; ++k) s[k] = cb0 + k < lim ? s[k] : -INFINITY;
            }
#pragma unroll
            for (int k = 0; k < 32; ++k) {
              const float2 a = fma2(make_float2(s[2 * k], s[2 * k + 1]), sc, off);
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
              float top[4] = {mx, x[0], x[1], x[2]};
#pragma unroll
              for (int k = 3; k < 32; ++k) top[k & 3] = fmaxf(top[k & 3], x[k]);
              mx = fmaxf(fmaxf(top[0], top[1]), fmaxf(top[2], top[3]));
            }
            mx *= scale_log2;
            const float up = (l < 0.5f * kMost ? mx : fmaxf(mx, ref)) + kRoom;   // a sum that has grown makes room too
            float f = 1.f;
            if (mine && up > ref) { f = ref == -INFINITY ? 0.f : fast_exp2(ref - up); ref = up; }
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
    }
    if (!ok) {
      c.err = 1;
      if (n_q > 0) wait_all(&c.q_full[e], (n_q - 1) & 1);         // no copy is in flight when the block ends
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

size_t paged_attn_tc_ws_bytes(const Paged& p, int group, int num_sms) {
  return paged_part_bytes(p, group, 2 * (kRows / group), num_sms);
}

int launch_paged_attn_tc(const Paged& p, int layer, int group, const void* q, void* out, int32_t* dev_status, void* ws,
                         int num_sms, cudaStream_t st) {
  static std::atomic<int> smem_set[64];
  int dev = 0;
  if (cudaGetDevice(&dev) != cudaSuccess || dev < 0 || dev >= 64 || smem_set[dev].load(std::memory_order_acquire) == 0) {
    if (cudaFuncSetAttribute(paged_attn_tc_kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)kSmemBytes) != cudaSuccess)
      return -1;
    if (dev >= 0 && dev < 64) smem_set[dev].store(1, std::memory_order_release);
  }
  CUtensorMap tmap, tmap_q;
  const int ps = 1 << p.page_log2;
  if (!make_tmap_rows_bf16(&tmap, p.pool + (int64_t)layer * p.layer_rows * kHeadDim * 2, (uint64_t)p.layer_rows, ps < kKeys ? ps : kKeys))
    return -1;
  if (!make_tmap_heads_bf16(&tmap_q, q, (uint32_t)(p.G * group), (uint64_t)p.T, (uint32_t)group, (uint32_t)(kRows / group))) return -1;
  unsigned char* w = static_cast<unsigned char*>(ws);
  Header* header = reinterpret_cast<Header*>(w);
  float* part = reinterpret_cast<float*>(w + kHeaderBytes);
  const int tq = kRows / group;
  if (!launch_pdl(paged_attn_tc_kernel, dim3(num_sms), kThreads, kSmemBytes, st, tmap, tmap_q, p, (__nv_bfloat16*)out, dev_status,
                  header, part, paged_part_rows(p, group, 2 * tq), paged_max_parts(num_sms), group,
                  kLog2e / sqrtf((float)kHeadDim)))
    return -1;
  return launch_paged_merge(p, group, out, dev_status, header, part, tq, 2 * tq, num_sms, st) < 0 ? -1 : 2;
}

}  // namespace vr
