// Paged attention: how a batch is cut into units, the same for every CTA and for the kernel that merges partials.
//
// A block is a run of bq new tokens of one sequence; a unit is (sequence, run of key tiles, block, KV head), units are
// numbered in that order. The length of a run is the same for the whole batch. Blocks of one sequence are taken longest first,
// and blocks that read the same keys stand next to each other, so that they meet in L2. Units of a block that is cut are
// partials: reference, sum and unnormalised values of their rows.
#pragma once

#include <math.h>

#include "common.cuh"
#include "paged.h"

namespace vr {

constexpr int kKeysBf16 = 128, kKeysF32 = 32;               // of a key tile: what a kernel takes at a time
constexpr int kCand = 32;
constexpr int kPartsPerSm = 4;                              // partial units that the workspace holds, per SM
constexpr int kNone = 0x7fff;                               // Ctl::special of the bf16 kernel: no such value

// Workspace: header, then the partials: values [rows][d], then (reference, sum) [rows].
struct Header {
  unsigned int taken;       // units taken from the counter; zero between calls
  unsigned int gave_up;     // a CTA timed out: not all units were taken; zero between calls
  int run, units, parts;    // key tiles of a run, units, and how many of them are partials
  int first;                // the number of units, from the take that found the counter at zero; zero between calls
  int open;                 // a call is between its start and the end of its merge; zero between calls
};
constexpr size_t kHeaderBytes = 256;
// Of a call that is two kernels: the second one's header, before the partials of any call on the same workspace.
constexpr size_t kSecondHeader = 128;
static_assert(sizeof(Header) <= kSecondHeader && kSecondHeader + sizeof(Header) <= kHeaderBytes, "two headers before the partials");

// A CTA's next unit, after its first one, which has its own number. At or past `units`: none, also where the counter was not
// zero before the call and is out of range. A counter found at c with 0 < c <= units - ctas ends at `units` like one found at
// zero (c units are skipped, and as many takes), so the merge looks for the take that got zero as well.
__device__ __forceinline__ int take_unit(Header* h, int ctas, int units) {
  const unsigned int t = atomicAdd(&h->taken, 1u);
  if (t == 0) h->first = units;
  return t < (unsigned int)units ? ctas + (int)t : units;
}

struct Unit {
  int valid, g, row0, ntok, pos0, t0, t1, e0, both, slot, values_from;
  // g: KV head; row0: row of the block's first token; pos0: its position; key tiles t0 .. t1 - 1, of which the first
  // warpgroup's query tile sees those before e0; both: one query tile for both; slot: partial, or -1; values_from: first
  // tile whose values have to be looked at
};
struct SeqUnit : Unit {     // where a kernel needs its sequence as well
  int seq;
};

// The sequences whose number of new tokens is in n_min .. n_max, of a batch that two kernels share.
struct PagedSome : Paged {
  int n_min, n_max;
};

// A sequence as a kernel's plan has it: without new tokens where it is another kernel's.
__device__ __forceinline__ bool plan_range(const Paged& p, int s, SeqRange& r) { return seq_range(p, s, r); }
__device__ __forceinline__ bool plan_range(const PagedSome& p, int s, SeqRange& r) {
  if (!seq_range(p, s, r)) return false;
  if (r.n < p.n_min || r.n > p.n_max) r.n = 0;
  return true;
}

// Key tiles that hold the first `keys` keys (keys < 2^32).
template <int kKeys>
__device__ __forceinline__ int tiles_of(uint32_t keys) { return (int)((keys + (kKeys - 1)) / kKeys); }

// Blocks, key tiles and cuts of one sequence.
struct SeqPlan {
  int row0, n, len, nb, tiles, cuts, chunk;
};
template <int kKeys>
__device__ __forceinline__ SeqPlan seq_plan(const SeqRange& r, int bq, int run) {
  SeqPlan q;
  q.row0 = r.row0; q.n = r.n; q.len = r.len;
  q.nb = (unsigned)(r.n + bq - 1) / (unsigned)bq;
  q.tiles = tiles_of<kKeys>(r.len);
  q.cuts = q.nb ? (unsigned)(q.tiles + run - 1) / (unsigned)run : 0;
  q.chunk = q.nb ? (unsigned)(q.tiles + q.cuts - 1) / (unsigned)q.cuts : 0;
  return q;
}

struct PlanSums {           // in shared memory, zero before plan_add
  int units[kCand], split[kCand], chunk[kCand];
};

// The length of a run of key tiles and the number of units. Weight W in tiles, C CTAs. A run of W (1 + i / 16) / (j C),
// j = 1..8, i = 0..3, or no cut: the shortest of what the last CTA takes, estimated as whole rounds of
// mean units and as an even share plus half of what the longest unit is above the mean; cuts that the workspace does
// not hold are left out. `overhead`: of a unit (start, output), in key tiles; `merge`, `part`: what merging takes, with a partial's share. Same for every CTA. Lane = candidate; the
// warps share the sequences and add up in plan_add, one warp decides in plan_choose.
template <int kKeys, typename P>
__device__ __forceinline__ float plan_weight(const P& p, int bq, int lane, int& longest) {
  float w = 0.f;
  int most = 0;
  for (int s = lane; s < p.S; s += 32) {
    SeqRange r;
    if (!plan_range(p, s, r) || r.n == 0) continue;
    const int last = tiles_of<kKeys>(r.len), first = tiles_of<kKeys>(r.len - r.n + min(bq, r.n));
    w += (float)((unsigned)(r.n + bq - 1) / (unsigned)bq) * (0.5f * (float)(first + last));
    most = max(most, last);
  }
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) {
    w += __shfl_xor_sync(0xffffffffu, w, o);
    most = max(most, __shfl_xor_sync(0xffffffffu, most, o));
  }
  longest = most;
  return w * (float)p.G;
}
__device__ __forceinline__ int plan_candidate(float W, int longest, int C, int lane) {
  if (lane == kCand - 1) return longest + 1;
  const float k = ceilf(W * (float)(16 + (lane & 3)) / (16.f * (float)(1 + (lane >> 2)) * (float)C));
  return min(max(1, (int)fminf(k, 1e9f)), longest + 1);
}
template <int kKeys, typename P>
__device__ __forceinline__ void plan_add(const P& p, PlanSums& c, int bq, int cand, int warp, int warps, int lane) {
  int u = 0, split = 0, chunk = 0;
  for (int s = warp; s < p.S; s += warps) {
    SeqRange r;
    if (!plan_range(p, s, r)) continue;
    const SeqPlan q = seq_plan<kKeys>(r, bq, cand);
    const int n = p.G * q.nb * q.cuts;
    u += n;
    split += q.cuts > 1 ? n : 0;
    chunk = max(chunk, q.chunk);
  }
  if (u) { atomicAdd(&c.units[lane], u); atomicAdd(&c.split[lane], split); atomicMax(&c.chunk[lane], chunk); }
}
__device__ __forceinline__ void plan_choose(const PlanSums& c, float W, int cand, int C, int max_parts, float overhead, int lane,
                                            int& run, int& units, int& parts, float merge = 0.f, float part = 0.f) {
  const int u = c.units[lane];
  float est = INFINITY;
  if (c.split[lane] <= max_parts) {
    const float total = W + overhead * (float)u, mean = total / fmaxf((float)u, 1.f);
    est = fmaxf(ceilf((float)u / C) * mean, total / C + 0.5f * fmaxf(0.f, (float)c.chunk[lane] + overhead - mean));
    if (merge > 0.f && c.split[lane]) est += merge + part * (float)c.split[lane] / C;
  }
  int best = lane;
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) {
    const float e = __shfl_xor_sync(0xffffffffu, est, o);
    const int b = __shfl_xor_sync(0xffffffffu, best, o);
    if (e < est || (e == est && b < best)) { est = e; best = b; }
  }
  run = __shfl_sync(0xffffffffu, cand, best);
  units = __shfl_sync(0xffffffffu, u, best);
  parts = c.split[best];
}

// Walks the units in increasing order; one warp. The lanes hold 32 sequences at a time.
template <int kKeys, typename P = Paged>
struct Walk {
  int s0 = 0, before = 0, parts_before = 0;     // first sequence held; units and partials before it
  int incl, parts_incl, total, parts;           // scans over the sequences held, and their sums
  SeqPlan q;

  __device__ __forceinline__ void load(const P& p, int bq, int run, int lane) {
    SeqRange r;
    r.n = 0; r.len = 0; r.row0 = 0;
    if (s0 + lane < p.S && !plan_range(p, s0 + lane, r)) r.n = 0;
    if (r.n == 0) r.len = 0;
    q = seq_plan<kKeys>(r, bq, run);
    incl = p.G * q.nb * q.cuts;
    parts_incl = q.cuts > 1 ? incl : 0;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const int y = __shfl_up_sync(0xffffffffu, incl, o), z = __shfl_up_sync(0xffffffffu, parts_incl, o);
      if (lane >= o) { incl += y; parts_incl += z; }
    }
    total = __shfl_sync(0xffffffffu, incl, 31);
    parts = __shfl_sync(0xffffffffu, parts_incl, 31);
  }
  __device__ __forceinline__ void next(const P& p, int bq, int run, int lane) {
    before += total;
    parts_before += parts;
    s0 += 32;
    load(p, bq, run, lane);
  }
  // unit u (at or after the last one asked for, below the number of units): its sequence and what it is
  __device__ __forceinline__ int find(const P& p, int bq, int tq, int run, int u, int lane, Unit& x) {
    while (u >= before + total && s0 < p.S) next(p, bq, run, lane);
    const int l = __ffs(__ballot_sync(0xffffffffu, u < before + incl)) - 1;
    if (l < 0) { x.valid = 0; x.t0 = 0; x.t1 = 0; return 0; }
    SeqPlan f;
    f.row0 = __shfl_sync(0xffffffffu, q.row0, l); f.n = __shfl_sync(0xffffffffu, q.n, l);
    f.len = __shfl_sync(0xffffffffu, q.len, l); f.nb = __shfl_sync(0xffffffffu, q.nb, l);
    f.cuts = __shfl_sync(0xffffffffu, q.cuts, l); f.chunk = __shfl_sync(0xffffffffu, q.chunk, l);
    const int units = p.G * f.nb * f.cuts;
    const int at = u - before - (__shfl_sync(0xffffffffu, incl, l) - units);
    const int gb = (unsigned)at / (unsigned)p.G, j = (unsigned)gb / (unsigned)f.nb, b = f.nb - 1 - (gb - j * f.nb);
    x.g = at - gb * p.G;
    x.ntok = min(bq, f.n - b * bq);
    x.row0 = f.row0 + b * bq;
    x.pos0 = f.len - f.n + b * bq;
    const int end = x.pos0 + x.ntok, tiles = tiles_of<kKeys>(end);
    x.t0 = j * f.chunk;
    x.t1 = min(x.t0 + f.chunk, tiles);
    x.both = x.ntok <= tq;
    x.e0 = max(x.t0, min(x.t1, tiles_of<kKeys>((uint32_t)x.pos0 + tq)));
    x.slot = f.cuts > 1 ? parts_before + __shfl_sync(0xffffffffu, parts_incl, l) - units + at : -1;
    x.values_from = max(x.t0, x.ntok > 1 ? (x.pos0 + 1) / kKeys : end / kKeys);
    x.valid = 1;
    return s0 + l;
  }
};

// Most partials that a workspace holds, and the rows of one.
inline int paged_max_parts(int num_sms) { return kPartsPerSm * num_sms; }
inline int paged_part_rows(const Paged& p, int group, int bq) {
  const int64_t rows = (int64_t)p.T * group, most = (int64_t)bq * group;
  return (int)(rows < most ? rows : most);
}
inline size_t paged_part_bytes(const Paged& p, int group, int bq, int num_sms) {
  const size_t rows = (size_t)paged_max_parts(num_sms) * paged_part_rows(p, group, bq);
  return kHeaderBytes + ((rows * (kHeadDim + 2) * sizeof(float) + 255) & ~size_t(255));
}
// Merges partials into `out` and leaves the header as the next call wants it. tq: tokens of a query tile, of which a block has
// one or two.
int launch_paged_merge(const Paged& p, int group, void* out, int32_t* dev_status, Header* header, const float* part, int tq,
                       int bq, int num_sms, cudaStream_t st);

}  // namespace vr
