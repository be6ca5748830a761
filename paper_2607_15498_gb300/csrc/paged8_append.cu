// Paged cache in 8 bits, append: head norm, rotation to the token's position, queries out, keys and values as codes into
// their pages, with a scale for each block of 16 tokens of a head.
//
// y = x / sqrt(mean(x^2) + eps) * w, the pairs (i, i + rot/2) turned by position * freq[i] (the angle in turns as a 64-bit
// integer, as in the append of the uncompressed cache), then for keys and values
//   byte = max(byte of the block's older tokens, least with max |z| <= 448 * 2^(byte - 127)),  code = e4m3(z / 2^(byte - 127)),
// and the older codes of the block times 2^(their byte - byte).
// A unit is a block of 16 places of one sequence that gets new tokens; a warp takes the 16 tokens of one of its H + 2 G heads:
// eight lanes a token, sixteen elements each (eight first members of pairs and their partners), four tokens at a time, so
// that a block's largest element is found by one warp. Sines and cosines of the 16 tokens are made once for the CTA's heads: those of every
// fourth token, and of the three behind it by a product with those of one, two and three positions (in units of 2^-24, off by 9 at most: the
// angles 1.6 each, their cosines and sines 1 each, times sqrt 2, and the product 1.2).
// Rows wait in shared memory as they came (cp.async), so that a thread holds no row that it does not work on and four CTAs fit
// an SM: with rows in registers and two CTAs the prompt below took 43 us.
//
// Bound by instructions and memory alike for prompts: 8192 tokens of 32 + 8 + 8 heads 36.7 us, 185 MB at 5.0 TB/s (0.74 of a
// copy); what is left is norm, turn, the largest element and two roundings a pair. 23 chunks of 30 to 900 tokens with norms, older
// tokens in their first blocks: 33.7 us, 104 MB at 0.45 of a copy. One token of eight sequences: 4.7 us, a launch and one chain of loads.
// On the way: sines and cosines of every token by themselves 38.7 us on that prompt (made once a CTA they would take it to 35.6).
#include "common.cuh"
#include "paged.h"
#include "paged8.h"

namespace vr {

namespace {

constexpr int kThreads = 256, kWarps = kThreads / 32, kCtas = 4;
constexpr int kSteps = kBlock / 4;            // a warp's rows of a task, four at a time

struct Append8Args {
  const __nv_bfloat16 *q, *k, *v, *q_norm, *k_norm;
  int64_t q_stride, k_stride, v_stride;
  const double* freq;
  const int32_t* gone;
  unsigned char *codes, *scale;               // of the layer
  float* mass;
  __nv_bfloat16* q_out;
  int32_t* dev_status;
  float eps;
  int rot, H, per;                            // H: 0 without queries; per: heads of an item
};

__device__ __forceinline__ void unpack(const uint4& u, float2 (&x)[4]) {
  const uint32_t w[4] = {u.x, u.y, u.z, u.w};
#pragma unroll
  for (int i = 0; i < 4; ++i) x[i] = make_float2(__uint_as_float(w[i] << 16), __uint_as_float(w[i] & 0xffff0000u));
}
__device__ __forceinline__ void load_pairs(const float* s, float2 (&x)[4]) {   // eight floats from shared memory
  const float4 a = reinterpret_cast<const float4*>(s)[0], b = reinterpret_cast<const float4*>(s)[1];
  x[0] = make_float2(a.x, a.y); x[1] = make_float2(a.z, a.w); x[2] = make_float2(b.x, b.y); x[3] = make_float2(b.z, b.w);
}
__device__ __forceinline__ float most(const float2 (&x)[4], float m) {
#pragma unroll
  for (int i = 0; i < 4; ++i) m = fmaxf(m, fmaxf(fabsf(x[i].x), fabsf(x[i].y)));
  return m;
}
// the largest of the finite ones (an infinity is stored as NaN)
__device__ __forceinline__ float most_finite(float2 (&x)[4], float m) {
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    if (fabsf(x[i].x) == INFINITY) x[i].x = NAN;
    if (fabsf(x[i].y) == INFINITY) x[i].y = NAN;
  }
  return most(x, m);
}
__device__ __forceinline__ uint2 codes8(const float2 (&x)[4], float f) {
  uint32_t c[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) c[i] = codes2(x[i].x * f, x[i].y * f);
  return make_uint2(c[0] | c[1] << 16, c[2] | c[3] << 16);
}

// Cosine and sine of a position times a frequency in turns, of which the upper 32 bits are kept: 2^-32 of a turn.
__device__ __forceinline__ void sine(unsigned long long turn, uint32_t pos, float& c, float& s) {
  const uint32_t at = (uint32_t)(turn >> 32) * pos + __umulhi((uint32_t)turn, pos);
  sincospif(__int2float_rn((int)at) * 0x1p-31f, &s, &c);
}

// Units of the sequences before s: more than there are, found without a sum over the sequences (n new tokens lie in at most
// (n + 14) / 16 + 1 <= n / 16 + 2 blocks).
__device__ __forceinline__ int first_unit(const int32_t* row_start, int s) { return (__ldg(row_start + s) >> kBlockLog2) + 2 * s; }

// The sequence whose units u is among: entries of first_unit[0 .. S] that are <= u, less one; one warp.
__device__ __forceinline__ int seq_of_unit(const Paged& p, int u, int lane) {
  int lo = 0, n = p.S + 1;
  while (n > 32) {
    const int step = (n + 31) >> 5, i = (lane + 1) * step - 1;
    const int k = __popc(__ballot_sync(0xffffffffu, i < n && first_unit(p.row_start, lo + i) <= u));
    lo += k * step;
    n = min(step, n - k * step);
  }
  return lo + __popc(__ballot_sync(0xffffffffu, lane < n && first_unit(p.row_start, lo + lane) <= u)) - 1;
}

__global__ void __launch_bounds__(kThreads, kCtas) paged8_append_kernel(Paged p, Append8Args a) {
  __shared__ unsigned long long turn[kHeadDim / 2];   // freq / 2 pi modulo 1, times 2^64
  __shared__ __align__(16) float weight[2][kHeadDim];
  __shared__ __align__(16) float angle[kBlock][2][kHeadDim / 2];   // of the item's tokens: cosines, sines
  __shared__ float step[3][2][kHeadDim / 2];           // of one, two and three positions
  __shared__ uint4 raw[kWarps][kSteps][2][32];                     // a warp's rows as they come, a lane's own
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, sub = lane & 7;
  pdl_trigger();
  pdl_wait();
  if (tid < a.rot / 2) {
    const double t = a.freq[tid] * 0.15915494309189535;   // 1 / 2 pi
    turn[tid] = __double2ull_rn((t - floor(t)) * 18446744073709551616.0);
  }
  if (const __nv_bfloat16* w = tid < kHeadDim ? a.q_norm : a.k_norm) weight[tid / kHeadDim][tid % kHeadDim] = __bfloat162float(w[tid % kHeadDim]);
  __syncthreads();
  const int tasks = a.H + 2 * p.G, chunks = (tasks + a.per - 1) / a.per, h8 = a.rot / 16;
  const int64_t items = (int64_t)((p.T >> kBlockLog2) + 2 * p.S + 1) * chunks;
  // this lane's two groups of eight elements: a group of first members and its partners, or two groups that stay
  const bool turns = sub < h8;
  const int e0 = 8 * (turns ? sub : sub + h8), e1 = 8 * (turns ? sub + h8 : sub + 8);

  bool stepped = false;                               // `step` is there
  for (int64_t it = blockIdx.x; it < items; it += gridDim.x) {
    const int u = (int)(it / chunks), lo = (int)(it % chunks) * a.per, hi = min(lo + a.per, tasks);
    const int s = seq_of_unit(p, u, lane);
    if (s < 0 || s >= p.S) continue;                  // (the same for the CTA)
    SeqRange r;
    if (!seq_range(p, s, r) || r.n == 0) continue;    // the status is raised below
    const int start = r.len - r.n;                    // place of the first new token
    const int64_t nth = (int64_t)u - first_unit(p.row_start, s), base64 = (((int64_t)start >> kBlockLog2) + nth) << kBlockLog2;
    if (nth < 0 || base64 >= r.len) continue;         // (below 0: row ranges out of order)
    const int base = (int)base64, old = max(start - base, 0), end = min(r.len - base, kBlock);   // new tokens: rows old .. end - 1
    const int row0 = r.row0 + (base - start);         // row of the block's first place
    int page = __ldg(p.table + (int64_t)s * p.max_pages + (base >> p.page_log2));
    const int gone = a.gone ? __ldg(a.gone + s) : 0;
    if (page < 0 || page >= p.n_pages || gone < 0) {
      if (tid == 0 && lo == 0) raise_status(a.dev_status, VARRATE_ERR_CORRUPT);
      if (gone < 0) continue;
      page = -1;
    }
    bool made = a.rot == 0;                           // the item's sines and cosines are there
    for (int t0 = lo; t0 < hi; t0 += kWarps) {
      const int task = t0 + warp;
      const bool is_q = task < a.H, is_v = task >= a.H + p.G, live = task < hi;
      const int row_in = lane >> 3;                   // of the first of this lane's four rows; the others are 4, 8 and 12 further
      int64_t code_row = 0;
      int before = 0;
      if (live) {
        const int64_t stride = is_q ? a.q_stride : is_v ? a.v_stride : a.k_stride;
        const __nv_bfloat16* src = is_q ? a.q + task * kHeadDim : is_v ? a.v + (task - a.H - p.G) * kHeadDim : a.k + (task - a.H) * kHeadDim;
        src += (row0 + row_in) * stride;
#pragma unroll
        for (int i = 0; i < kSteps; ++i) {            // rows that are none read as zeros
          const bool there = 4 * i + row_in >= old && 4 * i + row_in < end;
          const __nv_bfloat16* x = there ? src + 4 * i * stride : a.k;
          cp_async16(smem_addr(&raw[warp][i][0][lane]), x + e0, there ? 16 : 0);
          cp_async16(smem_addr(&raw[warp][i][1][lane]), x + e1, there ? 16 : 0);
        }
        if (!is_q && page >= 0) {
          code_row = page_row(p, page, is_v, task - a.H - (is_v ? p.G : 0), base & ((1 << p.page_log2) - 1));
          if (old) before = a.scale[scale_at(code_row)];
        }
      }
      cp_async_commit();
      if (!made) {                                    // behind the first loads
        __syncthreads();                              // (the last item's have been read)
        const int half = a.rot / 2;
        const bool single = end - old <= 4;           // each row by itself
        if (!single && !stepped) {
          for (int i = tid; i < 3 * half; i += kThreads) sine(turn[i % half], i / half + 1, step[i / half][0][i % half], step[i / half][1][i % half]);
          stepped = true;
          __syncthreads();
        }
        for (int i = tid; i < (single ? end - old : kBlock / 4) * half; i += kThreads) {
          const int j = i % half, row = single ? old + i / half : i / half * 4;
          float c0, s0;
          sine(turn[j], (uint32_t)base + row + gone, c0, s0);
          angle[row][0][j] = c0;
          angle[row][1][j] = s0;
          if (single) continue;
#pragma unroll
          for (int k = 1; k < 4; ++k) {
            const float c1 = step[k - 1][0][j], s1 = step[k - 1][1][j];
            angle[row + k][0][j] = fmaf(-s0, s1, c0 * c1);
            angle[row + k][1][j] = fmaf(c0, s1, s0 * c1);
          }
        }
        __syncthreads();
        made = true;
      }
      cp_async_wait<0>();
      if (!live || (!is_q && page < 0)) continue;
      const bool normed = is_q ? a.q_norm != nullptr : a.k_norm != nullptr && !is_v, turned = turns && !is_v;
      // Row i of this lane's four with its norm and rotation. Rows of keys and values are formed twice, for the scale and for the
      // codes, and read from shared memory each time: registers are the bound on the warps of an SM.
      auto form = [&](int i, float2 (&y0)[4], float2 (&y1)[4]) {
        const int row = 4 * i + row_in;
        unpack(raw[warp][i][0][lane], y0);
        unpack(raw[warp][i][1][lane], y1);
        if (normed) {                                 // (the same for the warp)
          float2 sq = make_float2(0.f, 0.f);
#pragma unroll
          for (int j = 0; j < 4; ++j) sq = fma2(y0[j], y0[j], fma2(y1[j], y1[j], sq));
          float ss = sq.x + sq.y;
#pragma unroll
          for (int o = 4; o > 0; o >>= 1) ss += __shfl_xor_sync(0xffffffffu, ss, o);
          const float f1 = row >= old && row < end ? rsqrtf(ss * (1.f / kHeadDim) + a.eps) : 0.f;
          const float2 f = make_float2(f1, f1);
          float2 w[4];
          load_pairs(weight[is_q ? 0 : 1] + e0, w);
#pragma unroll
          for (int j = 0; j < 4; ++j) y0[j] = mul2(mul2(y0[j], f), w[j]);
          load_pairs(weight[is_q ? 0 : 1] + e1, w);
#pragma unroll
          for (int j = 0; j < 4; ++j) y1[j] = mul2(mul2(y1[j], f), w[j]);
        }
        if (turned && row >= old && row < end) {
          float2 c[4], sn[4];
          load_pairs(angle[row][0] + e0, c);
          load_pairs(angle[row][1] + e0, sn);
#pragma unroll
          for (int j = 0; j < 4; ++j) {
            float2 z = mul2(y0[j], c[j]);               // (a product of pairs has no sign to turn)
            z = make_float2(fmaf(-y1[j].x, sn[j].x, z.x), fmaf(-y1[j].y, sn[j].y, z.y));
            y1[j] = fma2(y0[j], sn[j], mul2(y1[j], c[j]));
            y0[j] = z;
          }
        }
      };
      float2 y0[4], y1[4];
      if (is_q) {
        const bool copy = !normed && a.rot == 0;
        __nv_bfloat16* y = a.q_out + ((int64_t)(row0 + row_in) * a.H + task) * kHeadDim;
#pragma unroll 2
        for (int i = 0; i < kSteps; ++i) {
          uint4 z0, z1;
          if (copy) {
            z0 = raw[warp][i][0][lane];
            z1 = raw[warp][i][1][lane];
          } else {
            form(i, y0, y1);
            z0 = make_uint4(pack_bf16(y0[0].x, y0[0].y), pack_bf16(y0[1].x, y0[1].y), pack_bf16(y0[2].x, y0[2].y), pack_bf16(y0[3].x, y0[3].y));
            z1 = make_uint4(pack_bf16(y1[0].x, y1[0].y), pack_bf16(y1[1].x, y1[1].y), pack_bf16(y1[2].x, y1[2].y), pack_bf16(y1[3].x, y1[3].y));
          }
          if (4 * i + row_in < old || 4 * i + row_in >= end) continue;
          *reinterpret_cast<uint4*>(y + (int64_t)4 * i * a.H * kHeadDim + e0) = z0;
          *reinterpret_cast<uint4*>(y + (int64_t)4 * i * a.H * kHeadDim + e1) = z1;
        }
        continue;
      }
      float top = 0.f;
#pragma unroll 2
      for (int i = 0; i < kSteps; ++i) {
        form(i, y0, y1);
        top = most(y1, most(y0, top));
      }
      const bool odd = __any_sync(0xffffffffu, top == INFINITY);   // rare: infinities, which count as NaN
      if (odd) {
        top = 0.f;
#pragma unroll 1
        for (int i = 0; i < kSteps; ++i) {
          form(i, y0, y1);
          top = most_finite(y1, most_finite(y0, top));
        }
      }
#pragma unroll
      for (int o = 16; o > 0; o >>= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, o));
      const int byte = max(before, scale_byte(top));
      const float f = byte ? scale_inverse(byte) : 1.f;
      unsigned char* dst = a.codes + (code_row + row_in) * kHeadDim;
#pragma unroll 2
      for (int i = 0; i < kSteps; ++i) {
        const int row = 4 * i + row_in;
        uint2 *z0 = reinterpret_cast<uint2*>(dst + 4 * i * kHeadDim + e0), *z1 = reinterpret_cast<uint2*>(dst + 4 * i * kHeadDim + e1);
        form(i, y0, y1);
        if (odd) { most_finite(y0, 0.f); most_finite(y1, 0.f); }
        if (row < old) {
          if (byte != before) {
            const Rescale by(byte - before);
            const uint2 o0 = *z0, o1 = *z1;
            *z0 = make_uint2(by.four(o0.x), by.four(o0.y));
            *z1 = make_uint2(by.four(o1.x), by.four(o1.y));
          }
        } else if (row < end) {
          *z0 = codes8(y0, f);
          *z1 = codes8(y1, f);
        }
      }
      if (lane == 0) a.scale[scale_at(code_row)] = (unsigned char)byte;
      if (!is_v && a.mass && lane >= old && lane < end)
        a.mass[mass_at(p, page, task - a.H, (base & ((1 << p.page_log2) - 1)) + lane)] = 0.f;
    }
  }
  // every sequence's tables are checked, rows or not
  for (int s = blockIdx.x * kThreads + tid; s < p.S; s += gridDim.x * kThreads) {
    SeqRange r;
    if (!seq_range(p, s, r)) raise_status(a.dev_status, VARRATE_ERR_CORRUPT);
  }
}

}  // namespace

int launch_paged8_append(const Paged8& c, int layer, int group, const void* q, int64_t q_stride, const void* k,
                         int64_t k_stride, const void* v, int64_t v_stride, const void* q_norm, const void* k_norm,
                         float eps, const double* freq, int rot, const int32_t* gone, void* q_out, int32_t* dev_status,
                         int num_sms, cudaStream_t st) {
  const Paged& p = c.p;
  Append8Args a;
  a.q = (const __nv_bfloat16*)q; a.k = (const __nv_bfloat16*)k; a.v = (const __nv_bfloat16*)v;
  a.q_norm = q ? (const __nv_bfloat16*)q_norm : nullptr; a.k_norm = (const __nv_bfloat16*)k_norm;
  a.q_stride = q_stride; a.k_stride = k_stride; a.v_stride = v_stride;
  a.freq = freq; a.gone = gone; a.q_out = (__nv_bfloat16*)q_out; a.dev_status = dev_status; a.eps = eps; a.rot = rot;
  a.H = q ? group * p.G : 0;
  a.codes = p.pool + (int64_t)layer * p.layer_rows * kHeadDim;
  a.scale = c.scale + (int64_t)layer * (p.layer_rows >> kBlockLog2);
  a.mass = c.mass ? c.mass + (int64_t)layer * (p.layer_rows / 2) : nullptr;
  // whole units per CTA where there are enough of them, else their heads over several CTAs
  const int tasks = a.H + 2 * p.G;
  const int64_t units = (p.T >> kBlockLog2) + 2 * (int64_t)p.S + 1, most = (int64_t)num_sms * kCtas;
  a.per = (tasks + kWarps - 1) / kWarps * kWarps;
  while (a.per > kWarps && units * ((tasks + a.per - 1) / a.per) < 2 * most) a.per = (a.per / 2 + kWarps - 1) / kWarps * kWarps;
  const int64_t items = units * ((tasks + a.per - 1) / a.per);
  return launch_pdl(paged8_append_kernel, dim3((unsigned)(items < most ? items : most)), kThreads, 0, st, p, a) ? 1 : -1;
}

}  // namespace vr
