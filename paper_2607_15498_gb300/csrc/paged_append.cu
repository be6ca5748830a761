// Paged cache, append: head norm, rotation to the token's position, queries out, keys and values into their pages.
//
// Per head x (128 elements): y = x / sqrt(mean(x^2) + eps) * w, then the pairs (i, i + rot/2) turned by
// position * freq[i]. A half-warp holds one head, eight elements a lane: the mean square is four shuffles, the
// partner of a pair sits rot/16 lanes away. The angle is kept in turns: freq / 2 pi modulo 1 as a 64-bit integer F
// (one table per CTA, from doubles), so position * F mod 2^64 is the angle modulo a turn, exact up to the
// rounding of F however far the position, and its sine and cosine are taken once per token and warp.
// Bound by memory: every element is read and written once.
#include "common.cuh"
#include "paged.h"

namespace vr {

namespace {

constexpr int kThreads = 256;
constexpr int kWarps = kThreads / 32;
constexpr int kUnroll = 4;                 // heads in flight per half-warp
constexpr int kStep = 2 * kUnroll;         // heads per pass of a warp

__device__ __forceinline__ void load8(const float* p, float (&x)[8]) {
  const float4 a = __ldcs(reinterpret_cast<const float4*>(p)), b = __ldcs(reinterpret_cast<const float4*>(p) + 1);
  x[0] = a.x; x[1] = a.y; x[2] = a.z; x[3] = a.w; x[4] = b.x; x[5] = b.y; x[6] = b.z; x[7] = b.w;
}
__device__ __forceinline__ void load8(const __nv_bfloat16* p, float (&x)[8]) {
  const uint4 u = __ldcs(reinterpret_cast<const uint4*>(p));
  const uint32_t w[4] = {u.x, u.y, u.z, u.w};
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    x[2 * i] = __uint_as_float(w[i] << 16);
    x[2 * i + 1] = __uint_as_float(w[i] & 0xffff0000u);
  }
}
__device__ __forceinline__ void store8(float* p, const float (&x)[8]) {
  reinterpret_cast<float4*>(p)[0] = make_float4(x[0], x[1], x[2], x[3]);
  reinterpret_cast<float4*>(p)[1] = make_float4(x[4], x[5], x[6], x[7]);
}
__device__ __forceinline__ void store8(__nv_bfloat16* p, const float (&x)[8]) {
  *reinterpret_cast<uint4*>(p) = make_uint4(pack_bf16(x[0], x[1]), pack_bf16(x[2], x[3]), pack_bf16(x[4], x[5]),
                                            pack_bf16(x[6], x[7]));
}

// A warp takes `per` heads (a multiple of kStep) of one token: of its H query, G key and G value heads. q may be q_out.
template <typename T>
__global__ void __launch_bounds__(kThreads)
paged_append_kernel(Paged p, T* pool, const T* q, int64_t q_stride, const T* k, int64_t k_stride, const T* v,
                    int64_t v_stride, const T* __restrict__ q_norm, const T* __restrict__ k_norm, float eps,
                    const double* __restrict__ freq, int rot, T* q_out, int32_t* dev_status, int H, int per) {
  __shared__ unsigned long long turn[kHeadDim / 2];   // freq / 2 pi modulo 1, times 2^64
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, sub = lane & 15, half = lane >> 4;
  if (tid < rot / 2) {
    const double t = freq[tid] * 0.15915494309189535;   // 1 / 2 pi
    turn[tid] = __double2ull_rn((t - floor(t)) * 18446744073709551616.0);
  }
  __syncthreads();
  const int rows = H + 2 * p.G, chunks = (rows + per - 1) / per, h = rot / 2;
  const int64_t units = (int64_t)p.T * chunks;
  const int e0 = sub * 8;                             // this lane's elements of a head
  const bool first = e0 < h, turns = e0 < rot;
  const int partner = (lane & 16) | (turns ? (first ? sub + h / 8 : sub - h / 8) : sub);
  float wq[8], wk[8];
  if (q_norm) load8(q_norm + e0, wq);
  if (k_norm) load8(k_norm + e0, wk);

  // every sequence's tables are checked, rows or not
  for (int s = blockIdx.x * kThreads + tid; s < p.S; s += gridDim.x * kThreads) {
    SeqRange r;
    if (!seq_range(p, s, r)) raise_status(dev_status, VARRATE_ERR_CORRUPT);
  }
  for (int64_t u = (int64_t)blockIdx.x * kWarps + warp; u < units; u += (int64_t)gridDim.x * kWarps) {
    const int t = (int)(u / chunks), lo = (int)(u % chunks) * per, hi = min(lo + per, rows);
    const int s = count_le(p.row_start, p.S + 1, t, lane) - 1;
    if (s < 0 || s >= p.S) continue;                  // a row of no sequence
    SeqRange r;
    if (!seq_range(p, s, r) || t < r.row0 || t >= r.row0 + r.n) {
      raise_status(dev_status, VARRATE_ERR_CORRUPT);
      continue;
    }
    const int pos = r.len - r.n + (t - r.row0);
    const int page = __ldg(p.table + (int64_t)s * p.max_pages + (pos >> p.page_log2));
    const bool page_ok = page >= 0 && page < p.n_pages;
    if (!page_ok && lane == 0) raise_status(dev_status, VARRATE_ERR_CORRUPT);
    float c[8], sn[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      c[i] = 1.f;
      sn[i] = 0.f;
      if (turns) {
        const unsigned long long a = turn[(first ? e0 : e0 - h) + i] * (unsigned long long)pos;
        sincospif(__ll2float_rn((long long)a) * 0x1p-63f, &sn[i], &c[i]);
        if (first) sn[i] = -sn[i];
      }
    }
    for (int r0 = lo; r0 < hi; r0 += kStep) {
      float x[kUnroll][8];
#pragma unroll
      for (int i = 0; i < kUnroll; ++i) {
        const int row = r0 + 2 * i + half;
        if (row >= hi) continue;
        const T* src = row < H ? q + t * q_stride + row * kHeadDim
                     : row < H + p.G ? k + t * k_stride + (row - H) * kHeadDim
                                     : v + t * v_stride + (row - H - p.G) * kHeadDim;
        load8(src + e0, x[i]);
      }
#pragma unroll
      for (int i = 0; i < kUnroll; ++i) {
        const int row = r0 + 2 * i + half;
        const bool is_q = row < H, is_v = row >= H + p.G;
        float ss = 0.f;
#pragma unroll
        for (int j = 0; j < 8; ++j) ss = fmaf(x[i][j], x[i][j], ss);
#pragma unroll
        for (int o = 8; o > 0; o >>= 1) ss += __shfl_xor_sync(0xffffffffu, ss, o);
        if (!is_v && (is_q ? q_norm : k_norm) != nullptr) {
          const float f = rsqrtf(ss * (1.f / kHeadDim) + eps);
#pragma unroll
          for (int j = 0; j < 8; ++j) x[i][j] = x[i][j] * f * (is_q ? wq[j] : wk[j]);
        }
#pragma unroll
        for (int j = 0; j < 8; ++j) {
          const float y = __shfl_sync(0xffffffffu, x[i][j], partner);
          if (turns && !is_v) x[i][j] = fmaf(y, sn[j], x[i][j] * c[j]);
        }
        if (row >= hi) continue;
        if (is_q) {
          store8(q_out + ((int64_t)t * H + row) * kHeadDim + e0, x[i]);
        } else if (page_ok) {
          const int g = is_v ? row - H - p.G : row - H;
          store8(pool + page_row(p, page, is_v, g, pos & ((1 << p.page_log2) - 1)) * kHeadDim + e0, x[i]);
        }
      }
    }
  }
}

template <typename T>
int launch(const Paged& p, int layer, int group, const void* q, int64_t q_stride, const void* k, int64_t k_stride,
           const void* v, int64_t v_stride, const void* q_norm, const void* k_norm, float eps, const double* freq,
           int rot, void* q_out, int32_t* dev_status, int num_sms, cudaStream_t st) {
  const int H = q ? group * p.G : 0, rows = H + 2 * p.G;
  // whole tokens per warp where there are enough of them, else their heads over several warps
  int per = (rows + kStep - 1) / kStep * kStep;
  while (per > kStep && (int64_t)p.T * ((rows + per - 1) / per) < (int64_t)num_sms * kWarps) per = (per / 2 + kStep - 1) / kStep * kStep;
  const int64_t units = (int64_t)p.T * ((rows + per - 1) / per);
  const int64_t ctas = (units + kWarps - 1) / kWarps;
  const int grid = (int)(ctas < (int64_t)num_sms * 8 ? ctas : (int64_t)num_sms * 8);
  T* pool = reinterpret_cast<T*>(p.pool) + (int64_t)layer * p.layer_rows * kHeadDim;
  paged_append_kernel<T><<<grid, kThreads, 0, st>>>(p, pool, (const T*)q, q_stride, (const T*)k, k_stride, (const T*)v,
                                                    v_stride, (const T*)q_norm, (const T*)k_norm, eps, freq, rot,
                                                    (T*)q_out, dev_status, H, per);
  return 1;
}

}  // namespace

int launch_paged_append(const Paged& p, int layer, int group, const void* q, int64_t q_stride, const void* k,
                        int64_t k_stride, const void* v, int64_t v_stride, const void* q_norm, const void* k_norm,
                        float eps, const double* freq, int rot, void* q_out, int32_t* dev_status, int num_sms,
                        cudaStream_t st) {
  return p.dtype == VARRATE_F32
             ? launch<float>(p, layer, group, q, q_stride, k, k_stride, v, v_stride, q_norm, k_norm, eps, freq, rot,
                             q_out, dev_status, num_sms, st)
             : launch<__nv_bfloat16>(p, layer, group, q, q_stride, k, k_stride, v, v_stride, q_norm, k_norm, eps, freq,
                                     rot, q_out, dev_status, num_sms, st);
}

}  // namespace vr
