// Paged cache in 8 bits, attention weight of every cached token, sequences of many new tokens: tcgen05 products with the keys as rows.
//
// A unit is 256 keys of a sequence and KV head, in two tiles of 128, with every row that sees them:
//   S[key][row] = K[key][.] Q[row][.]     M = 128, N = 128, K = 128,
//   mass[key] += sum over rows of 2^(S scale - log2 e lse[row]).
// The keys stay, expanded to bf16 (exact, with the block's scale) in TMEM, and the queries of 128 rows at a time go past them; both key tiles
// use every query tile. (With the keys in shared memory its bandwidth was the bound: 64 KB a product of 512 cycles.) Two threads of
// the four epilogue warpgroups have a key, each half of the rows of a query tile, and add up in registers, so a token's sum has one
// order and is added to its mass once. Rows of a query tile are (token, head) pairs, tq = 128 / group tokens.
//
// Warps: 0-3, 4-7 sums of a key tile each over the first 64 rows, 8-11, 12-15 over the others; 16 TMA producer; 17, 18 issue the
// products of a key tile each; 19 fetches log2 e lse; 20-23 expand keys, a thread a key.
// Bound by the exponentials and the additions beside the products: 512 tokens on 130560, 32 heads over 8: 379 us, 550 GFLOP at 1450 TFLOP/s
// (0.76 of the measured bf16 rate). 2.15 10^9 exponentials take 230 us of the special function units if nothing waits, the
// adding and scaling instructions nearly as long beside them; a unit's start and end take 1.6 us of its 14.
// On the way: keys in shared memory 606 us, in TMEM 573; the lse of a query tile fetched one tile ahead instead of when it is needed
// 418, two ahead and its place found without divisions 396; keys expanded before the last unit is done, both barriers of a tile
// looked at together and the registers split 379. With the scores' place given back before they are added it is 385 to 426: the two
// key tiles' warps then take the special function units at the same time.
//
// Units are dealt out in turns, back and forth, the first of a sequence (which most rows see) first. Every wait is bounded; one
// that gives up raises VARRATE_ERR_TIMEOUT and its CTA ends after its copies and products in flight have.
#include <math.h>
#include <stddef.h>

#include <atomic>

#include <cudaTypedefs.h>

#include "common.cuh"
#include "decode_common.cuh"
#include "paged.h"
#include "paged8.h"
#include "paged8_mma.cuh"
#include "paged8_tc.cuh"

namespace vr {

bool make_tmap_rows_u8(CUtensorMap* map, const void* base, uint64_t rows, uint32_t box_rows);
bool make_tmap_heads_bf16(CUtensorMap* map, const void* base, uint32_t heads, uint64_t rows, uint32_t box_heads, uint32_t box_rows);

namespace {

constexpr int kThreads = 768;
constexpr int kSumWarps = 16, kProducer = 16, kIssuer = 17, kRowsWarp = 19, kExpand = 20;   // issuers: 17 and 18
// Registers a thread by warpgroup, four of sums, producer to lse, expansion: 4 * 88 + 56 + 72 = 6 * 80 of the launch.
constexpr int kSumRegs = 88, kOtherRegs = 56, kExpandRegs = 72;
constexpr int kTile = 128, kPair = 2 * kTile;               // keys of a tile, of a unit
constexpr int kTileBytes = kTile * kHeadDim * 2;
constexpr int kCodeBytes = kTile * kHeadDim;
constexpr int kQueries = 5, kLse = 4, kUnits = 4;           // query tiles, rows of lse and units in flight
constexpr int kScores = 3;                                  // score tiles in TMEM, 128 columns each; behind them the keys, 64 a tile

struct MassUnit {
  int valid, seq, g, key0, row0, n, len, q0, q1;            // row0: row of the sequence's first new token; query tiles q0 .. q1 - 1
};

struct Shared {
  unsigned char codes[2][2][kCodeBytes];                    // [unit & 1][tile]
  unsigned char query[kQueries][kTileBytes];
  float lse[kLse][kTile];                                   // -log2 e lse of a query tile's rows; -infinity where one adds nothing
  uint64_t raw[2][2], raw_empty[2][2], k_full[2], k_empty[2], q_full[kQueries], q_empty[kQueries], e_full[kLse], e_empty[kLse];
  uint64_t s_full[2][4], s_done[2][4];                      // of a key tile's score tiles, by their number
  uint64_t half_full[2][kUnits];                            // by the unit: the second half's warps may be two ahead of the first's
  uint64_t u_full[kUnits], u_empty[kUnits], drain[2];
  MassUnit unit[kUnits];
  int dead[kLse];                                           // some row of the tile adds nothing
  int err;
  uint32_t tmem;
};
static_assert(sizeof(Shared) <= 232448, "shared memory of a block");

// Both at once: a wait for what is there already takes as long as it takes to look.
__device__ __forceinline__ bool warp_wait_both(uint64_t* a, uint32_t pa, uint64_t* b, uint32_t pb) {
  for (uint32_t i = 0; i < kWaitTries; ++i) {
    const bool x = mbar_try_wait(a, pa), y = mbar_try_wait(b, pb);
    if (__all_sync(0xffffffffu, x & y)) return true;
  }
  return false;
}
__device__ __forceinline__ void tmem_st1(uint32_t taddr, float v) {
  asm volatile("tcgen05.st.sync.aligned.32x32b.x1.b32 [%0], {%1};\n" ::"r"(taddr), "f"(v) : "memory");
}
__device__ __forceinline__ float tmem_ld1(uint32_t taddr) {
  float v;
  asm volatile("tcgen05.ld.sync.aligned.32x32b.x1.b32 {%0}, [%1];\n tcgen05.wait::ld.sync.aligned;\n" : "=f"(v) : "r"(taddr) : "memory");
  return v;
}

__global__ void __launch_bounds__(kThreads, 1)
paged8_mass_tc_kernel(const __grid_constant__ CUtensorMap tmap, const __grid_constant__ CUtensorMap tmap_q, Paged p,
                      const unsigned char* __restrict__ scale, float* __restrict__ mass, const float* __restrict__ lse,
                      int32_t* __restrict__ dev_status, int grp, int few, float scale_log2) {
  extern __shared__ __align__(1024) unsigned char smem[];
  Shared& c = *reinterpret_cast<Shared*>(smem);
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const int tq = kTile / grp, H = p.G * grp, C = gridDim.x;
  if (tid == 0) {
    for (int i = 0; i < 2; ++i) {
      mbar_init(&c.k_full[i], 4); mbar_init(&c.k_empty[i], 1);
      for (int j = 0; j < 2; ++j) { mbar_init(&c.raw[i][j], 1); mbar_init(&c.raw_empty[i][j], 4); }
    }
    for (int i = 0; i < 4; ++i)
      for (int j = 0; j < 2; ++j) { mbar_init(&c.s_full[j][i], 1); mbar_init(&c.s_done[j][i], 8); }
    for (int i = 0; i < kQueries; ++i) { mbar_init(&c.q_full[i], 1); mbar_init(&c.q_empty[i], 2); }
    for (int i = 0; i < kLse; ++i) { mbar_init(&c.e_full[i], 1); mbar_init(&c.e_empty[i], kSumWarps); }
    for (int i = 0; i < kUnits; ++i) {
      mbar_init(&c.u_full[i], 1); mbar_init(&c.u_empty[i], kSumWarps + 3 + 4);
      for (int j = 0; j < 2; ++j) mbar_init(&c.half_full[j][i], 4);
    }
    for (int i = 0; i < 2; ++i) mbar_init(&c.drain[i], 1);
    c.err = 0;
    fence_mbar_init();
  }
  // rows of a query tile past tq * grp are never written again: their scores are of no row, but numbers
  for (int i = tid; i < kQueries * kTileBytes / 16; i += kThreads) reinterpret_cast<uint4*>(c.query)[i] = make_uint4(0, 0, 0, 0);
  fence_proxy_async_smem();
  if (warp == kIssuer) tmem_alloc(&c.tmem, 512);
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tmem = c.tmem;
  pdl_trigger();
  pdl_wait();
  bool some = false;                                          // a sequence for this kernel, or it ends here
  for (int s = tid; s < p.S; s += kThreads) {
    SeqRange r;
    some |= seq_range(p, s, r) && r.n > few;
  }
  if (!__syncthreads_or(some)) {
    if (warp == kIssuer) tmem_dealloc(tmem, 512);
    return;
  }

  if (warp >= kExpand) {
    fewer_registers<kExpandRegs>();
    // ------------------------------------------------------------------ codes to bf16: one key per thread
    const int key_in = tid - 32 * kExpand;
    bool ok = true;
    for (uint32_t un = 0; ok; ++un) {
      ok = warp_wait(&c.u_full[un % kUnits], (un / kUnits) & 1);
      if (!ok) break;
      const MassUnit x = c.unit[un % kUnits];
      __syncwarp();
      if (!x.valid) break;
      if (lane == 0) mbar_arrive(&c.u_empty[un % kUnits]);
      uint32_t byte[2] = {0, 0};
#pragma unroll
      for (int e = 0; e < 2; ++e) {
        const int key = x.key0 + e * kTile + key_in;
        if (key >= x.len) continue;
        const int page = __ldg(p.table + (int64_t)x.seq * p.max_pages + (key >> p.page_log2));
        if (page >= 0 && page < p.n_pages) byte[e] = __ldg(scale + scale_at(page_row(p, page, 0, x.g, key & ((1 << p.page_log2) - 1))));
      }
#pragma unroll 1
      for (int e = 0; e < 2; ++e) {
        ok = ok && warp_wait(&c.raw[un & 1][e], (un >> 1) & 1);
        if (!ok) break;
        const unsigned char* row = c.codes[un & 1][e] + key_in * 128;
        const uint32_t scale2 = (e ? byte[1] : byte[0]) * 0x00800080u, to = tmem + kScores * kTile + 64 * e + ((uint32_t)((warp & 3) * 32) << 16);
        const bool there = x.key0 + e * kTile + key_in < x.len;
        uint4 y[4][4];                                            // expanded while the last unit's products run
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          uint4 w = *reinterpret_cast<const uint4*>(row + ((i ^ (key_in & 7)) << 4));
          if (!there) w = make_uint4(0, 0, 0, 0);
          expand16(w, scale2, y[i >> 1][2 * (i & 1)], y[i >> 1][2 * (i & 1) + 1]);
        }
        __syncwarp();
        if (lane == 0) mbar_arrive(&c.raw_empty[un & 1][e]);
        ok = warp_wait(&c.k_empty[e], (un & 1) ^ 1);
        if (!ok) break;
        tc_fence_after();
#pragma unroll
        for (int h = 0; h < 4; ++h) tmem_st16(to + 16 * h, reinterpret_cast<const uint32_t(&)[16]>(y[h]));   // 32 elements
        tmem_wait_st();
        tc_fence_before();
        __syncwarp();
        if (lane == 0) mbar_arrive(&c.k_full[e]);
      }
    }
    if (!ok) c.err = 1;
  } else if (warp >= kSumWarps) {
    fewer_registers<kOtherRegs>();
    if (warp == kProducer) {
      // ------------------------------------------------------------------ units, keys and queries
      // Units of the 32 sequences from s0 on: [sequence][pair of tiles][head].
      int s0 = 0, k = 0;
      int64_t before = 0, incl = 0, total = 0;
      SeqRange r;
      auto scan = [&]() {
        incl = 0;
        if (s0 + lane < p.S && seq_range(p, s0 + lane, r) && r.n > few) incl = (int64_t)((r.len + kPair - 1) / kPair) * p.G;
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
          const int64_t y = __shfl_up_sync(0xffffffffu, incl, o);
          if (lane >= o) incl += y;
        }
        total = __shfl_sync(0xffffffffu, incl, 31);
      };
      scan();
      auto next_unit = [&]() {                                      // the CTA's k-th
        const int64_t u = (int64_t)k * C + (k & 1 ? C - 1 - (int)blockIdx.x : (int)blockIdx.x);
        ++k;
        MassUnit x = {};
        while (u >= before + total && s0 < p.S) {
          before += total;
          s0 += 32;
          scan();
        }
        if (u >= before + total) return x;
        const int l = __ffs(__ballot_sync(0xffffffffu, u < before + incl)) - 1;
        x.len = __shfl_sync(0xffffffffu, r.len, l);
        x.n = __shfl_sync(0xffffffffu, r.n, l);
        x.row0 = __shfl_sync(0xffffffffu, r.row0, l);
        const int64_t units = (int64_t)((x.len + kPair - 1) / kPair) * p.G, at = u - (before + __shfl_sync(0xffffffffu, incl, l) - units);
        const int pair = (int)(at / p.G);
        x.g = (int)(at - (int64_t)pair * p.G);
        x.key0 = pair * kPair;
        x.seq = s0 + l;
        x.q0 = max(0, x.key0 - (x.len - x.n)) / tq;
        x.q1 = (int)((unsigned)(x.n + tq - 1) / (unsigned)tq);
        x.valid = 1;
        return x;
      };
      const int page_keys = min(1 << p.page_log2, kTile), per_tile = kTile / page_keys;
      uint32_t nu = 0, nq = 0, nk = 0;                              // units published, query tiles and pairs of key tiles asked for
      bool ok = true;
      auto publish = [&](const MassUnit& x) {
        if (!warp_wait(&c.u_empty[nu % kUnits], ((nu / kUnits) & 1) ^ 1)) return false;
        if (lane == 0) {
          c.unit[nu % kUnits] = x;
          mbar_arrive(&c.u_full[nu % kUnits]);
        }
        ++nu;
        return true;
      };
      auto keys = [&](const MassUnit& x) {
        const uint32_t slot = nk & 1, fill = nk >> 1;
        for (int e = 0; e < 2; ++e)
          if (!warp_wait(&c.raw_empty[slot][e], (fill & 1) ^ 1)) return false;
        ++nk;
        for (int e = 0; e < 2; ++e) {
          const int base = x.key0 + e * kTile, key = base + lane * page_keys;
          const int boxes = max(0, min(per_tile, (x.len - base + page_keys - 1) / page_keys));
          if (lane == 0) mbar_arrive_expect_tx(&c.raw[slot][e], (uint32_t)boxes * page_keys * 128);
          __syncwarp();
          if (lane < boxes) {
            int page = __ldg(p.table + (int64_t)x.seq * p.max_pages + (key >> p.page_log2));
            if (page < 0 || page >= p.n_pages) {
              raise_status(dev_status, VARRATE_ERR_CORRUPT);
              page = 0;
            }
            tma_load_2d(smem_addr(c.codes[slot][e]) + lane * page_keys * 128, &tmap, 0,
                        (int)page_row(p, page, 0, x.g, key & ((1 << p.page_log2) - 1)), &c.raw[slot][e]);
          }
        }
        __syncwarp();
        return true;
      };
      MassUnit x = next_unit();
      ok = publish(x) && (!x.valid || keys(x));
      while (ok && x.valid) {
        MassUnit y = {};
        for (int t = x.q0; t < x.q1 && ok; ++t) {
          if (t == min(x.q0 + kQueries, x.q1 - 1)) {                // the next unit's keys, behind the first queries
            y = next_unit();
            ok = publish(y) && (!y.valid || keys(y));
            if (!ok) break;
          }
          const uint32_t slot = nq % kQueries;
          ok = warp_wait(&c.q_empty[slot], ((nq / kQueries) & 1) ^ 1);
          if (!ok) break;
          ++nq;
          if (lane == 0) {
            mbar_arrive_expect_tx(&c.q_full[slot], (uint32_t)(tq * grp) * 256);
            for (int half = 0; half < 2; ++half)
              tma_load_3d(smem_addr(c.query[slot]) + half * (kTile * 128), &tmap_q, half * 64, x.g * grp, x.row0 + t * tq, &c.q_full[slot]);
          }
          __syncwarp();
        }
        x = y;
      }
      if (!ok) {                                                    // no copy is in flight when the block ends
        c.err = 1;
        for (uint32_t i = nq > kQueries ? nq - kQueries : 0; i < nq; ++i) warp_wait(&c.q_full[i % kQueries], (i / kQueries) & 1);
        for (uint32_t i = nk > 2 ? nk - 2 : 0; i < nk; ++i)
          for (int e = 0; e < 2; ++e) warp_wait(&c.raw[i & 1][e], (i >> 1) & 1);
      }
    } else if (warp == kIssuer || warp == kIssuer + 1) {
      // ------------------------------------------------------------------ products of key tile e
      // (values that are the same in every lane, broadcast from lane 0 where they come from memory, stay in uniform registers)
      constexpr uint32_t idesc = idesc_bf16_f32(kTile, kTile);
      const int e = __shfl_sync(0xffffffffu, warp - kIssuer, 0);
      const uint32_t tm = __shfl_sync(0xffffffffu, tmem, 0), keys = tm + kScores * kTile + 64 * e;
      const uint64_t queries = sdesc_sw128(smem_addr(c.query));
      uint32_t slot = 0, q_phase = 0, at = e, n = 0;                // of the next query tile; where its scores go; its number
      bool ok = true;
      for (uint32_t un = 0; ok; ++un) {
        ok = warp_wait(&c.u_full[un % kUnits], (un / kUnits) & 1);
        if (!ok) break;
        const MassUnit* x = &c.unit[un % kUnits];
        const int valid = __shfl_sync(0xffffffffu, x->valid, 0), tiles = __shfl_sync(0xffffffffu, x->q1 - x->q0, 0);
        if (!valid) break;
        if (lane == 0) mbar_arrive(&c.u_empty[un % kUnits]);
        ok = warp_wait(&c.k_full[e], un & 1);
        for (int t = 0; t < tiles && ok; ++t) {
          ok = warp_wait(&c.q_full[slot], q_phase);
          // the scores' place: of the two key tiles' products, taken in turn, it was that of the third before this one, of the other tile
          const uint32_t m = n + e - 2;
          if (ok && n + e >= 2) ok = warp_wait(&c.s_done[e ^ 1][m & 3], (m >> 2) & 1);
          if (!ok) break;
          tc_fence_after();
          if (elect_one()) {
            const uint64_t q = queries + slot * (kTileBytes / 16);
#pragma unroll
            for (int ks = 0; ks < kHeadDim / 16; ++ks)
              tc_mma_bf16_ts(tm + at * kTile, keys + 8 * ks, q + ((ks >> 2) * (kTile * 128) + (ks & 3) * 32) / 16, idesc, ks != 0);
            tc_commit(&c.s_full[e][n & 3]);
            tc_commit(&c.q_empty[slot]);
            if (t == tiles - 1) tc_commit(&c.k_empty[e]);
          }
          __syncwarp();
          if (++slot == kQueries) { slot = 0; q_phase ^= 1; }
          at = at + 2 >= kScores ? at + 2 - kScores : at + 2;
          ++n;
        }
      }
      if (!ok) {                                                    // the products in flight end before TMEM is freed
        c.err = 1;
        if (elect_one()) tc_commit(&c.drain[e]);
        warp_wait(&c.drain[e], 0);
      }
      __syncwarp();
    } else if (warp == kRowsWarp) {
      // ------------------------------------------------------------------ log2 e lse of the rows
      uint32_t n = 0;
      bool ok = true;
      int token[4], off[4];                                         // of this lane's rows of a tile: past every tile's where there is none
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const int row = lane + 32 * i;
        token[i] = row < tq * grp ? row / grp : INT32_MAX / 2;
        off[i] = row / grp * H + row % grp;
      }
      for (uint32_t un = 0; ok; ++un) {
        ok = warp_wait(&c.u_full[un % kUnits], (un / kUnits) & 1);
        if (!ok) break;
        const MassUnit x = c.unit[un % kUnits];
        __syncwarp();
        if (!x.valid) break;
        if (lane == 0) mbar_arrive(&c.u_empty[un % kUnits]);
        float z[2][4];                                              // lse of the next two tiles' rows
        auto fetch = [&](int t, float (&z)[4]) {
#pragma unroll
          for (int i = 0; i < 4; ++i)
            z[i] = t < x.q1 && token[i] < x.n - t * tq ? __ldg(lse + (int64_t)(x.row0 + t * tq) * H + x.g * grp + off[i]) : 0.f;
        };
        fetch(x.q0, z[0]);
        fetch(x.q0 + 1, z[1]);
        for (int t0 = x.q0; t0 < x.q1 && ok; t0 += 2) {
#pragma unroll
          for (int h = 0; h < 2; ++h) {
            const int t = t0 + h;
            if (t >= x.q1 || !ok) break;
            float y[4];
            bool dead = false;
#pragma unroll
            for (int i = 0; i < 4; ++i) {
              const bool there = token[i] < x.n - t * tq, finite = fabsf(z[h][i]) < INFINITY;
              y[i] = there && finite ? -z[h][i] * kLog2e : -INFINITY;
              dead |= there && !finite;
            }
            dead = __any_sync(0xffffffffu, dead);
            fetch(t + 2, z[h]);
            ok = warp_wait(&c.e_empty[n % kLse], ((n / kLse) & 1) ^ 1);
            if (!ok) break;
#pragma unroll
            for (int i = 0; i < 4; ++i) c.lse[n % kLse][lane + 32 * i] = y[i];
            if (lane == 0) c.dead[n % kLse] = dead;
            __syncwarp();
            if (lane == 0) mbar_arrive(&c.e_full[n % kLse]);
            ++n;
          }
        }
      }
      if (!ok) c.err = 1;
    }
  } else {
    more_registers<kSumRegs>();
    // ------------------------------------------------------------------ sums: one key per thread
    const int e = warp >> 2 & 1, half = warp >> 3, r = tid & 127;
    const uint32_t lanes = (uint32_t)((warp & 3) * 32) << 16;
    uint32_t n = 0;
    bool ok = true;
    for (uint32_t un = 0; ok; ++un) {
      ok = warp_wait(&c.u_full[un % kUnits], (un / kUnits) & 1);
      if (!ok) break;
      const MassUnit x = c.unit[un % kUnits];
      __syncwarp();
      if (!x.valid) break;
      if (lane == 0) mbar_arrive(&c.u_empty[un % kUnits]);
      const int key = x.key0 + e * kTile + r, ahead = key - (x.len - x.n);   // the first new token that sees the key
      const int page = key < x.len ? __ldg(p.table + (int64_t)x.seq * p.max_pages + (key >> p.page_log2)) : -1;
      const int top = __shfl_sync(0xffffffffu, ahead, 31);
      float2 sum[2] = {make_float2(0.f, 0.f), make_float2(0.f, 0.f)};
      float total = 0.f;
      for (int t = x.q0; t < x.q1; ++t, ++n) {
        const uint32_t at = (2 * n + e) % kScores, slot = n % kLse, ts = tmem + at * kTile + lanes;
        ok = warp_wait_both(&c.e_full[slot], (n / kLse) & 1, &c.s_full[e][n & 3], (n >> 2) & 1);
        if (!ok) break;
        tc_fence_after();
        // some key of the warp is behind some row of the tile, or the tile has rows that add nothing
        const bool cut = top > t * tq || (t + 1) * tq > x.n || c.dead[slot];
        const int lo = max(0, ahead - t * tq) * grp, hi = min(tq, x.n - t * tq) * grp;
        float2 part[2] = {make_float2(0.f, 0.f), make_float2(0.f, 0.f)};
        const uint32_t mine = ts + 64 * half;
        const float* less = c.lse[slot] + 64 * half;
        if (cut) {
#pragma unroll 1
          for (int cb = 0; cb < 64; cb += 32) {
            float s[32];
            tmem_ld32(mine + cb, s);
#pragma unroll
            for (int k = 0; k < 32; ++k) {
              const int col = 64 * half + cb + k;
              const float l = less[cb + k];
              s[k] = col >= lo && col < hi && l > -INFINITY ? fmaf(s[k], scale_log2, l) : -INFINITY;
            }
#pragma unroll
            for (int k = 0; k < 16; ++k) part[k & 1] = add2(part[k & 1], make_float2(fast_exp2(s[2 * k]), fast_exp2(s[2 * k + 1])));
          }
        } else {
          const float2 sc = make_float2(scale_log2, scale_log2);
          float s0[32], s1[32];
          auto add = [&](float (&s)[32], const float* l) {
#pragma unroll
            for (int k = 0; k < 8; ++k) {
              const float4 y = reinterpret_cast<const float4*>(l)[k];
              const float2 u = fma2(make_float2(s[4 * k], s[4 * k + 1]), sc, make_float2(y.x, y.y));
              const float2 v = fma2(make_float2(s[4 * k + 2], s[4 * k + 3]), sc, make_float2(y.z, y.w));
              part[0] = add2(part[0], make_float2(fast_exp2(u.x), fast_exp2(u.y)));
              part[1] = add2(part[1], make_float2(fast_exp2(v.x), fast_exp2(v.y)));
            }
          };
          tmem_ld32_async(mine, s0);
          tmem_wait_ld32(s0);
          tmem_ld32_async(mine + 32, s1);                         // under the sum of the first
          add(s0, less);
          tmem_wait_ld32(s1);
          add(s1, less + 32);
        }
        sum[0] = add2(sum[0], part[0]);
        sum[1] = add2(sum[1], part[1]);
        if (t == x.q1 - 1) {                                      // the two halves meet in the scores' place
          const float2 w = add2(sum[0], sum[1]);
          total = w.x + w.y;
          if (half) {
            tmem_st1(ts + 64, total);
            tmem_wait_st();
            tc_fence_before();
            __syncwarp();
            if (lane == 0) mbar_arrive(&c.half_full[e][un % kUnits]);
          } else {
            ok = warp_wait(&c.half_full[e][un % kUnits], (un / kUnits) & 1);
            if (!ok) break;
            tc_fence_after();
            total += tmem_ld1(ts + 64);
          }
        }
        tc_fence_before();
        __syncwarp();
        if (lane == 0) {
          mbar_arrive(&c.s_done[e][n & 3]);
          mbar_arrive(&c.e_empty[slot]);
        }
      }
      if (!ok) break;
      // one addition to a token in a call: the order is no matter
      if (!half && page >= 0 && page < p.n_pages) atomicAdd(mass + mass_at(p, page, x.g, key & ((1 << p.page_log2) - 1)), total);
    }
    if (!ok) c.err = 1;
  }
  __syncthreads();
  if (warp == kIssuer) tmem_dealloc(tmem, 512);
  if (tid == 0 && c.err) raise_status(dev_status, VARRATE_ERR_TIMEOUT);
}

}  // namespace

int launch_paged8_mass_tc(const Paged8& c, int layer, int group, const void* q, const float* lse, int32_t* dev_status,
                          int num_sms, cudaStream_t st) {
  const Paged& p = c.p;
  static std::atomic<int> smem_set[64];
  int dev = 0;
  if (cudaGetDevice(&dev) != cudaSuccess || dev < 0 || dev >= 64 || smem_set[dev].load(std::memory_order_acquire) == 0) {
    if (!registers_for(paged8_mass_tc_kernel, kThreads, 128 * (4 * kSumRegs + kOtherRegs + kExpandRegs))) return -1;
    if (cudaFuncSetAttribute(paged8_mass_tc_kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)sizeof(Shared)) != cudaSuccess) return -1;
    if (dev >= 0 && dev < 64) smem_set[dev].store(1, std::memory_order_release);
  }
  CUtensorMap tmap, tmap_q;
  const int ps = 1 << p.page_log2;
  if (!make_tmap_rows_u8(&tmap, p.pool + (int64_t)layer * p.layer_rows * kHeadDim, (uint64_t)p.layer_rows, ps < kTile ? ps : kTile)) return -1;
  if (!make_tmap_heads_bf16(&tmap_q, q, (uint32_t)(p.G * group), (uint64_t)p.T, (uint32_t)group, (uint32_t)(kTile / group))) return -1;
  return launch_pdl(paged8_mass_tc_kernel, dim3(num_sms), kThreads, sizeof(Shared), st, tmap, tmap_q, p,
                    c.scale + (int64_t)layer * (p.layer_rows >> kBlockLog2), c.mass + (int64_t)layer * (p.layer_rows / 2), lse,
                    dev_status, group, few_tokens(p, group), kLog2e / sqrtf((float)kHeadDim))
             ? 1 : -1;
}

}  // namespace vr
