// Paged cache in 8 bits, attention weight of every cached token, sequences of many new tokens: tcgen05 products with the keys as rows.
//
// A unit is 256 keys of a sequence and KV head, in two tiles of 128, with every row that sees them:
//   S[key][row] = K[key][.] Q[row][.]     M = 128, N = 128, K = 128,
//   mass[key] += sum over rows of 2^(S scale - log2 e lse[row]).
// The keys stay, expanded to bf16 (exact, with the block's scale), and the queries of 128 rows at a time go past them; both key tiles use every
// query tile. A thread of the two epilogue warpgroups has a key and adds up in registers, so a token's sum has one order and is added to
// its mass once. Rows of a query tile are (token, head) pairs, tq = 128 / group tokens.
//
// Warps: 0-3, 4-7 sums of a key tile each; 8 TMA producer; 9 issues products; 10 fetches log2 e lse; 12-15 expand keys, a thread a key.
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

constexpr int kThreads = 512;
constexpr int kSumWarps = 8, kProducer = 8, kIssuer = 9, kRowsWarp = 10, kExpand = 12;
constexpr int kTile = 128, kPair = 2 * kTile;               // keys of a tile, of a unit
constexpr int kTileBytes = kTile * kHeadDim * 2;
constexpr int kQueries = 3, kLse = 4, kUnits = 4;           // query tiles, rows of lse and units in flight

struct MassUnit {
  int valid, seq, g, key0, row0, n, len, q0, q1;            // row0: row of the sequence's first new token; query tiles q0 .. q1 - 1
};

struct Shared {
  unsigned char keys[2][2][kTileBytes];                     // [unit & 1][tile]
  unsigned char query[kQueries][kTileBytes];
  float lse[kLse][kTile];                                   // log2 e lse of a query tile's rows; infinity where one adds nothing
  uint64_t raw[2][2], k_full[2][2], k_empty[2], q_full[kQueries], q_empty[kQueries], e_full[kLse], e_empty[kLse];
  uint64_t s_full[2][2], s_empty[2][2], u_full[kUnits], u_empty[kUnits], drain;
  MassUnit unit[kUnits];
  int dead[kLse];                                           // some row of the tile adds nothing
  int err;
  uint32_t tmem;
};
static_assert(sizeof(Shared) <= 232448, "shared memory of a block");

__global__ void __launch_bounds__(kThreads, 1)
paged8_mass_tc_kernel(const __grid_constant__ CUtensorMap tmap, const __grid_constant__ CUtensorMap tmap_q, Paged p,
                      const unsigned char* __restrict__ scale, float* __restrict__ mass, const float* __restrict__ lse,
                      int32_t* __restrict__ dev_status, int grp, int few, float scale_log2) {
  extern __shared__ __align__(1024) unsigned char smem[];
  Shared& c = *reinterpret_cast<Shared*>(smem);
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const int tq = kTile / grp, H = p.G * grp, C = gridDim.x;
  pdl_trigger();
  if (tid == 0) {
    for (int i = 0; i < 2; ++i) {
      mbar_init(&c.k_empty[i], 1);
      for (int j = 0; j < 2; ++j) {
        mbar_init(&c.raw[i][j], 1); mbar_init(&c.k_full[i][j], 4); mbar_init(&c.s_full[i][j], 1); mbar_init(&c.s_empty[i][j], 4);
      }
    }
    for (int i = 0; i < kQueries; ++i) { mbar_init(&c.q_full[i], 1); mbar_init(&c.q_empty[i], 1); }
    for (int i = 0; i < kLse; ++i) { mbar_init(&c.e_full[i], 1); mbar_init(&c.e_empty[i], kSumWarps); }
    for (int i = 0; i < kUnits; ++i) { mbar_init(&c.u_full[i], 1); mbar_init(&c.u_empty[i], kSumWarps + 2 + 4); }
    mbar_init(&c.drain, 1);
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
  __threadfence();   // the kernel before this one takes other sequences, and lets this one start when what comes before both has ended

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
      const uint32_t slot = nk & 1;
      if (!warp_wait(&c.k_empty[slot], ((nk >> 1) & 1) ^ 1)) return false;
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
          tma_load_2d(smem_addr(c.keys[slot][e]) + kTile * 128 + lane * page_keys * 128, &tmap, 0,
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
  } else if (warp == kIssuer) {
    // ------------------------------------------------------------------ products
    constexpr uint32_t idesc = idesc_bf16_f32(kTile, kTile);
    const uint32_t tm = __shfl_sync(0xffffffffu, tmem, 0), keys = smem_addr(c.keys), queries = smem_addr(c.query);
    uint32_t n = 0;                                               // query tiles so far
    bool ok = true;
    for (uint32_t un = 0; ok; ++un) {
      ok = warp_wait(&c.u_full[un % kUnits], (un / kUnits) & 1);
      if (!ok) break;
      const MassUnit* x = &c.unit[un % kUnits];
      const int valid = __shfl_sync(0xffffffffu, x->valid, 0), tiles = __shfl_sync(0xffffffffu, x->q1 - x->q0, 0);
      if (!valid) break;
      if (lane == 0) mbar_arrive(&c.u_empty[un % kUnits]);
      for (int t = 0; t < tiles && ok; ++t, ++n) {
        const uint32_t slot = n % kQueries, b = n & 1;
        ok = warp_wait(&c.q_full[slot], (n / kQueries) & 1);
#pragma unroll
        for (int e = 0; e < 2; ++e) {
          if (ok && t == 0) ok = warp_wait(&c.k_full[un & 1][e], (un >> 1) & 1);
          ok = ok && warp_wait(&c.s_empty[e][b], ((n >> 1) & 1) ^ 1);
          if (!ok) break;
          tc_fence_after();
          if (elect_one()) {
            const uint64_t a = sdesc_sw128(keys + ((un & 1) * 2 + e) * kTileBytes), q = sdesc_sw128(queries + slot * kTileBytes);
#pragma unroll
            for (int ks = 0; ks < kHeadDim / 16; ++ks) {
              const uint64_t o = (uint64_t)((ks >> 2) * (kTile * 128) + (ks & 3) * 32) / 16;
              tc_mma_bf16(tm + (2 * e + b) * kTile, a + o, q + o, idesc, ks != 0);
            }
            tc_commit(&c.s_full[e][b]);
            if (e == 1) {
              tc_commit(&c.q_empty[slot]);
              if (t == tiles - 1) tc_commit(&c.k_empty[un & 1]);
            }
          }
          __syncwarp();
        }
      }
    }
    if (!ok) {                                                    // the products in flight end before TMEM is freed
      c.err = 1;
      if (elect_one()) tc_commit(&c.drain);
      warp_wait(&c.drain, 0);
    }
    __syncwarp();
  } else if (warp == kRowsWarp) {
    // ------------------------------------------------------------------ log2 e lse of the rows
    uint32_t n = 0;
    bool ok = true;
    for (uint32_t un = 0; ok; ++un) {
      ok = warp_wait(&c.u_full[un % kUnits], (un / kUnits) & 1);
      if (!ok) break;
      const MassUnit x = c.unit[un % kUnits];
      __syncwarp();
      if (!x.valid) break;
      if (lane == 0) mbar_arrive(&c.u_empty[un % kUnits]);
      for (int t = x.q0; t < x.q1; ++t, ++n) {
        float y[4];
        bool dead = false;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const int row = lane + 32 * i, tok = t * tq + row / grp;
          y[i] = INFINITY;
          if (row >= tq * grp || tok >= x.n) continue;
          const float z = __ldg(lse + (int64_t)(x.row0 + tok) * H + x.g * grp + row % grp);
          if (fabsf(z) < INFINITY) y[i] = z * kLog2e;
          else dead = true;
        }
        dead = __any_sync(0xffffffffu, dead);
        ok = warp_wait(&c.e_empty[n % kLse], ((n / kLse) & 1) ^ 1);
        if (!ok) break;
#pragma unroll
        for (int i = 0; i < 4; ++i) c.lse[n % kLse][lane + 32 * i] = y[i];
        if (lane == 0) c.dead[n % kLse] = dead;
        __syncwarp();
        if (lane == 0) mbar_arrive(&c.e_full[n % kLse]);
      }
    }
    if (!ok) c.err = 1;
  } else if (warp >= kExpand) {
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
#pragma unroll
      for (int e = 0; e < 2; ++e) {
        ok = ok && warp_wait(&c.raw[un & 1][e], (un >> 1) & 1);
        if (!ok) break;
        expand_row<true>(c.keys[un & 1][e], kTile, key_in, x.key0 + e * kTile + key_in < x.len, byte[e]);
        fence_proxy_async_smem();
        __syncwarp();
        if (lane == 0) mbar_arrive(&c.k_full[un & 1][e]);
      }
    }
    if (!ok) c.err = 1;
  } else if (warp < kSumWarps) {
    // ------------------------------------------------------------------ sums: one key per thread
    const int e = warp >> 2, r = tid & 127;
    const uint32_t ts = tmem + 2 * e * kTile + ((uint32_t)((warp & 3) * 32) << 16);
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
      for (int t = x.q0; t < x.q1; ++t, ++n) {
        const uint32_t b = n & 1, slot = n % kLse;
        ok = warp_wait(&c.e_full[slot], (n / kLse) & 1) && warp_wait(&c.s_full[e][b], (n >> 1) & 1);
        if (!ok) break;
        tc_fence_after();
        // some key of the warp is behind some row of the tile, or the tile has rows that add nothing
        const bool cut = top > t * tq || (t + 1) * tq > x.n || c.dead[slot];
        const int lo = max(0, ahead - t * tq) * grp, hi = min(tq, x.n - t * tq) * grp;
        float2 part[2] = {make_float2(0.f, 0.f), make_float2(0.f, 0.f)};
#pragma unroll 1
        for (int cb = 0; cb < kTile; cb += 64) {
          float s[64];
          tmem_ld64(ts + b * kTile + cb, s);
          const float4* y = reinterpret_cast<const float4*>(c.lse[slot] + cb);
          if (cut) {
#pragma unroll
            for (int k = 0; k < 16; ++k) {
              const float4 l4 = y[k];
              const float l[4] = {l4.x, l4.y, l4.z, l4.w};
#pragma unroll
              for (int j = 0; j < 4; ++j) {
                const int col = cb + 4 * k + j;
                s[4 * k + j] = col >= lo && col < hi && l[j] < INFINITY ? fmaf(s[4 * k + j], scale_log2, -l[j]) : -INFINITY;
              }
            }
          } else {
            const float2 sc = make_float2(scale_log2, scale_log2);
#pragma unroll
            for (int k = 0; k < 16; ++k) {
              const float4 l = y[k];
              const float2 u = fma2(make_float2(s[4 * k], s[4 * k + 1]), sc, make_float2(-l.x, -l.y));
              const float2 v = fma2(make_float2(s[4 * k + 2], s[4 * k + 3]), sc, make_float2(-l.z, -l.w));
              s[4 * k] = u.x; s[4 * k + 1] = u.y; s[4 * k + 2] = v.x; s[4 * k + 3] = v.y;
            }
          }
#pragma unroll
          for (int k = 0; k < 32; ++k) part[k & 1] = add2(part[k & 1], make_float2(fast_exp2(s[2 * k]), fast_exp2(s[2 * k + 1])));
        }
        tc_fence_before();
        __syncwarp();
        if (lane == 0) {
          mbar_arrive(&c.s_empty[e][b]);
          mbar_arrive(&c.e_empty[slot]);
        }
        sum[0] = add2(sum[0], part[0]);
        sum[1] = add2(sum[1], part[1]);
      }
      if (!ok) break;
      const float2 w = add2(sum[0], sum[1]);
      // one addition to a token in a call: the order is no matter
      if (page >= 0 && page < p.n_pages) atomicAdd(mass + mass_at(p, page, x.g, key & ((1 << p.page_log2) - 1)), w.x + w.y);
    }
    if (!ok) c.err = 1;
  }
  __syncthreads();
  if (warp == kIssuer) tmem_dealloc(tmem, 512);
  if (tid == 0 && c.err) raise_status(dev_status, VARRATE_ERR_TIMEOUT);
  pdl_wait();                                                 // so that what waits for this kernel waits for both
}

}  // namespace

int launch_paged8_mass_tc(const Paged8& c, int layer, int group, const void* q, const float* lse, int32_t* dev_status,
                          int num_sms, cudaStream_t st) {
  const Paged& p = c.p;
  static std::atomic<int> smem_set[64];
  int dev = 0;
  if (cudaGetDevice(&dev) != cudaSuccess || dev < 0 || dev >= 64 || smem_set[dev].load(std::memory_order_acquire) == 0) {
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
