// Paged attention in 8 bits: the partials of blocks that were cut, merged.
#include "common.cuh"
#include "paged.h"
#include "paged8.h"
#include "paged_plan.cuh"

namespace vr {

namespace {

// A warp per (row, query head); a lane has four columns. A run of a block counts for a row only where the row's query tile
// reaches it. kBatch runs are read at once, merged with the running reference and sum: eight where every row has a warp of its own
// at two CTAs an SM (single tokens), else four at four CTAs. A chunk of 383 tokens, with its attention, 49.5 us for 51.4 with eight; one
// token on 8000 17.2 for 14.9. Which of the two kernels took a row's sequence, and so which plan and partials are its own, follows
// from the number of the sequence's new tokens.
// Bound by latency: what a row needs is read in two steps, first headers and tables, then its partials. 2.5 us of the 10.4 of a
// step over 900 tokens. Where nothing was cut (a prompt) it ends after the headers.
template <int kBatch, int kCtas>
__global__ void __launch_bounds__(256, kCtas)
paged8_merge_kernel(Paged p, __nv_bfloat16* __restrict__ out, int32_t* dev_status, unsigned char* first, int tq1, int part_rows1,
                    Merge8 two, int part_rows2, int max_parts, int grp) {
  constexpr int kKeys = kKeysBf16;
  const unsigned lane = threadIdx.x & 31, warp = threadIdx.x >> 5, H = p.G * grp;
  pdl_trigger();
  pdl_wait();
  const Header h1 = *reinterpret_cast<Header*>(first);
  Header h2 = {};
  if (two.second) h2 = *reinterpret_cast<Header*>(first + kSecondHeader);
  const unsigned total = (unsigned)p.T * H;                       // rows of 128 elements: below 2^31
  const bool any = h1.parts != 0 || h2.parts != 0;
  for (unsigned i = blockIdx.x * 8 + warp; any && i < total; i += gridDim.x * 8) {
    const int t = (int)(i / H), hq = (int)(i - (unsigned)t * H);
    const int s = count_le(p.row_start, p.S + 1, t, (int)lane) - 1;
    SeqRange r;
    if (s < 0 || s >= p.S || !seq_range(p, s, r) || t < r.row0 || t >= r.row0 + r.n) continue;
    const bool few = r.n <= two.few;
    const Header h = few ? h1 : h2;
    if (h.parts == 0) continue;
    const float* const part = few ? reinterpret_cast<const float*>(first + kHeaderBytes) : two.second;
    const int part_rows = few ? part_rows1 : part_rows2, tq = few ? tq1 : two.tq2, bq = few ? tq1 : 2 * two.tq2;
    const float2* const ml = reinterpret_cast<const float2*>(part + (int64_t)max_parts * part_rows * kHeadDim);
    const SeqPlan f = seq_plan<kKeys>(r, bq, h.run);
    if (f.cuts < 2) continue;
    int before = 0;                                               // partials of the sequences before this one
    for (int s0 = 0; s0 < s; s0 += 32) {
      SeqRange r1;
      if (s0 + (int)lane < s && seq_range(p, s0 + lane, r1) && (r1.n <= two.few) == few) {
        const SeqPlan f1 = seq_plan<kKeys>(r1, bq, h.run);
        before += f1.cuts > 1 ? p.G * f1.nb * f1.cuts : 0;
      }
    }
    if (s > 0) {
#pragma unroll
      for (int o = 16; o > 0; o >>= 1) before += __shfl_xor_sync(0xffffffffu, before, o);
    }
    const int g = hq / (unsigned)grp, tok = t - f.row0, b = (unsigned)tok / (unsigned)bq, in = tok - b * bq, ntok = min(bq, f.n - b * bq);
    // the row's query tile: its last token's position decides which runs it reaches
    const int last = ntok <= tq ? ntok : in < tq ? tq : ntok;
    const int runs = (unsigned)(tiles_of<kKeys>(f.len - f.n + b * bq + last) + f.chunk - 1) / (unsigned)f.chunk;
    const int64_t slot = before + (int64_t)(f.nb - 1 - b) * p.G + g, slots = (int64_t)f.nb * p.G;   // first one, from run to run
    if (slot < 0 || slot + (runs - 1) * slots >= max_parts) {     // the header is another call's
      if (lane == 0) raise_status(dev_status, VARRATE_ERR_CORRUPT);
      continue;
    }
    const int64_t row0 = slot * part_rows + in * grp + (hq - g * grp);
    const int64_t step = slots * part_rows;
    // a part's weights sum to 1 at most: with this factor, a power of two that cancels, those of all parts do
    const float room = __int_as_float((127 - (32 - __clz(runs - 1))) << 23);
    float m = -INFINITY, l = 0.f;
    float4 v = make_float4(0.f, 0.f, 0.f, 0.f);
    for (int j0 = 0; j0 < runs; j0 += kBatch) {
      float2 x[kBatch];
      float4 y[kBatch];
#pragma unroll
      for (int j = 0; j < kBatch; ++j) {
        x[j] = make_float2(-INFINITY, 0.f);
        y[j] = make_float4(0.f, 0.f, 0.f, 0.f);
        if (j0 + j < runs) {
          x[j] = __ldcg(ml + row0 + (j0 + j) * step);
          y[j] = __ldcg(reinterpret_cast<const float4*>(part + (row0 + (j0 + j) * step) * kHeadDim) + lane);
        }
      }
      float top = m;
#pragma unroll
      for (int j = 0; j < kBatch; ++j) top = fmaxf(top, x[j].x);
      const float ref = top == -INFINITY ? 0.f : top, f0 = fast_exp2(m - ref);
      m = top;
      l *= f0;
      v.x *= f0; v.y *= f0; v.z *= f0; v.w *= f0;
#pragma unroll
      for (int j = 0; j < kBatch; ++j) {
        const float w = fast_exp2(x[j].x - ref) * room;
        l = fmaf(x[j].y, w, l);
        v.x = fmaf(y[j].x, w, v.x); v.y = fmaf(y[j].y, w, v.y); v.z = fmaf(y[j].z, w, v.z); v.w = fmaf(y[j].w, w, v.w);
      }
    }
    const float f1 = l == 0.f ? 0.f : 1.f / l;
    *reinterpret_cast<uint2*>(out + (int64_t)i * kHeadDim + lane * 4) = make_uint2(pack_bf16(v.x * f1, v.y * f1), pack_bf16(v.z * f1, v.w * f1));
    if (two.lse && lane == 0)                                     // (less what makes room)
      two.lse[i] = l == 0.f ? -INFINITY : (m + log2f(l) + (float)(32 - __clz(runs - 1))) * 0.69314718f;
  }
  auto close = [&](unsigned char* ws, const Header& h) {
    Header* const header = reinterpret_cast<Header*>(ws);
    if ((h.taken != (unsigned)h.units || h.first != h.units) && !h.gave_up) raise_status(dev_status, VARRATE_ERR_CORRUPT);
    header->taken = 0;
    header->gave_up = 0;
    header->first = 0;
    header->open = 0;
  };
  if (blockIdx.x == 0 && threadIdx.x == 0) {
    close(first, h1);
    if (two.second) close(first + kSecondHeader, h2);
  }
}

}  // namespace

int launch_paged8_merge(const Paged& p, int group, void* out, int32_t* dev_status, void* ws, int tq, const Merge8& two,
                        int num_sms, cudaStream_t st) {
  const int64_t warps = (int64_t)p.T * p.G * group;
  const unsigned grid = (unsigned)(warps < (int64_t)num_sms * 32 ? (warps + 7) / 8 : (int64_t)num_sms * 4);
  return launch_pdl(warps <= (int64_t)num_sms * 16 ? paged8_merge_kernel<8, 1> : paged8_merge_kernel<4, 4>, dim3(grid), 256, 0, st, p, (__nv_bfloat16*)out, dev_status, (unsigned char*)ws, tq,
                    paged_part_rows(p, group, tq), two, paged_part_rows(p, group, 2 * two.tq2), paged_max_parts(num_sms), group)
             ? 1 : -1;
}

}  // namespace vr
