// Paged attention: the partials of blocks that were cut, merged.
#include "common.cuh"
#include "paged.h"
#include "paged_plan.cuh"

namespace vr {

namespace {

__device__ __forceinline__ void store4(__nv_bfloat16* p, float4 v) {
  *reinterpret_cast<uint2*>(p) = make_uint2(pack_bf16(v.x, v.y), pack_bf16(v.z, v.w));
}
__device__ __forceinline__ void store4(float* p, float4 v) { *reinterpret_cast<float4*>(p) = v; }

// A warp per (row, query head); a lane has four columns. A run of a block counts for a row only where the row's query tile
// reaches it. Eight runs are read at once, merged with the running reference and sum.
// Bound by latency: what a row needs is read in two steps, first header and tables, then its partials.
template <typename T>
__global__ void __launch_bounds__(256)
paged_attn_merge_kernel(Paged p, T* __restrict__ out, int32_t* dev_status, Header* header, const float* __restrict__ part,
                        int part_rows, int max_parts, int grp, int tq, int bq) {
  constexpr int kBatch = 8, kKeys = sizeof(T) == 4 ? kKeysF32 : kKeysBf16;
  const unsigned lane = threadIdx.x & 31, warp = threadIdx.x >> 5, H = p.G * grp;
  pdl_trigger();
  pdl_wait();
  const Header h = *header;
  const float2* ml = reinterpret_cast<const float2*>(part + (int64_t)max_parts * part_rows * kHeadDim);
  const unsigned total = (unsigned)p.T * H;                       // rows of 128 elements: below 2^31
  for (unsigned i = blockIdx.x * 8 + warp; i < total; i += gridDim.x * 8) {
    const int t = (int)(i / H), hq = (int)(i - (unsigned)t * H);
    const int s = count_le(p.row_start, p.S + 1, t, (int)lane) - 1;
    SeqRange r;
    if (s < 0 || s >= p.S || !seq_range(p, s, r) || t < r.row0 || t >= r.row0 + r.n) continue;
    if (h.parts == 0) break;
    const SeqPlan f = seq_plan<kKeys>(r, bq, h.run);
    if (f.cuts < 2) continue;
    int before = 0;                                               // partials of the sequences before this one
    for (int s0 = 0; s0 < s; s0 += 32) {
      SeqRange r1;
      if (s0 + (int)lane < s && seq_range(p, s0 + lane, r1)) {
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
    store4(out + (int64_t)i * kHeadDim + lane * 4, make_float4(v.x * f1, v.y * f1, v.z * f1, v.w * f1));
  }
  if (blockIdx.x == 0 && threadIdx.x == 0) {
    if ((h.taken != (unsigned)h.units || h.first != h.units) && !h.gave_up) raise_status(dev_status, VARRATE_ERR_CORRUPT);
    header->taken = 0;
    header->gave_up = 0;
    header->first = 0;
    header->open = 0;
  }
}

template <typename T>
int launch(const Paged& p, int group, void* out, int32_t* dev_status, Header* header, const float* part, int tq, int bq,
           int num_sms, cudaStream_t st) {
  const int64_t warps = (int64_t)p.T * p.G * group;
  const unsigned grid = (unsigned)(warps < (int64_t)num_sms * 32 ? (warps + 7) / 8 : (int64_t)num_sms * 4);
  return launch_pdl(paged_attn_merge_kernel<T>, dim3(grid), 256, 0, st, p, (T*)out, dev_status, header, part,
                    paged_part_rows(p, group, bq), paged_max_parts(num_sms), group, tq, bq)
             ? 1 : -1;
}

}  // namespace

int launch_paged_merge(const Paged& p, int group, void* out, int32_t* dev_status, Header* header, const float* part, int tq,
                       int bq, int num_sms, cudaStream_t st) {
  return p.dtype == VARRATE_F32 ? launch<float>(p, group, out, dev_status, header, part, tq, bq, num_sms, st)
                                : launch<__nv_bfloat16>(p, group, out, dev_status, header, part, tq, bq, num_sms, st);
}

}  // namespace vr
