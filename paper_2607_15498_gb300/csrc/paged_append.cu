// Paged cache, append: head norm, rotation to the token's position, queries out, keys and values into their pages.
//
// Per head x (128 elements): y = x / sqrt(mean(x^2) + eps) * w, then the pairs (i, i + rot/2) turned by
// position * freq[i]. Eight lanes hold a head, sixteen elements each: for i < rot/2 eight first members of pairs and
// their eight partners, so that a rotation needs no other lane; the mean square is three shuffles. The angle is kept in
// turns: freq / 2 pi modulo 1 as a 64-bit integer F (one table per CTA, from doubles), so position * F mod 2^64 is the
// angle modulo a turn, exact up to the rounding of F however far the position; a warp takes sines and cosines once per
// token, two a lane.
// Bound by memory: every element is read and written once. 8192 tokens of 32 + 8 + 8 heads, bf16: 37 us, 5.5 TB/s (80 % of a
// copy); 32770 tokens of 28 + 4 + 4 heads with norms: 115 us, 5.2 TB/s. Sixteen warps an SM with sixteen heads in flight
// each, all of them resident (with eight CTAs an SM 38 and 122). More in flight is not faster: 24 warps take 50 us on the
// first, copies to shared memory two steps ahead 38, an L2 prefetch of the next token changes nothing. Stores that are
// evicted first would take 36, but the attention that follows reads what they write. A head on 16 lanes that exchange the
// pairs by shuffles: 94 us.
#include "common.cuh"
#include "paged.h"

namespace vr {

namespace {

constexpr int kThreads = 256;
constexpr int kWarps = kThreads / 32;
constexpr int kHeads = 4;                  // heads of a warp's step
template <typename T> constexpr int kCtas = sizeof(T) == 2 ? 2 : 3;   // per SM

// Eight elements as they are stored.
template <typename T> struct Raw { uint4 u[sizeof(T) / 2]; };

template <typename T>
__device__ __forceinline__ Raw<T> load_raw(const T* p) {   // (q may be q_out: no read-only loads)
  Raw<T> r;
#pragma unroll
  for (int i = 0; i < (int)sizeof(T) / 2; ++i) r.u[i] = reinterpret_cast<const uint4*>(p)[i];
  return r;
}
template <typename T>
__device__ __forceinline__ void store_raw(T* p, const Raw<T>& r) {
#pragma unroll
  for (int i = 0; i < (int)sizeof(T) / 2; ++i) reinterpret_cast<uint4*>(p)[i] = r.u[i];
}
// as four pairs of floats, for the packed arithmetic
__device__ __forceinline__ void unpack(const Raw<float>& r, float2 (&x)[4]) {
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    x[2 * i] = make_float2(__uint_as_float(r.u[i].x), __uint_as_float(r.u[i].y));
    x[2 * i + 1] = make_float2(__uint_as_float(r.u[i].z), __uint_as_float(r.u[i].w));
  }
}
__device__ __forceinline__ void unpack(const Raw<__nv_bfloat16>& r, float2 (&x)[4]) {
  const uint32_t w[4] = {r.u[0].x, r.u[0].y, r.u[0].z, r.u[0].w};
#pragma unroll
  for (int i = 0; i < 4; ++i) x[i] = make_float2(__uint_as_float(w[i] << 16), __uint_as_float(w[i] & 0xffff0000u));
}
__device__ __forceinline__ void pack(const float2 (&x)[4], Raw<float>& r) {
#pragma unroll
  for (int i = 0; i < 2; ++i)
    r.u[i] = make_uint4(__float_as_uint(x[2 * i].x), __float_as_uint(x[2 * i].y), __float_as_uint(x[2 * i + 1].x),
                        __float_as_uint(x[2 * i + 1].y));
}
__device__ __forceinline__ void pack(const float2 (&x)[4], Raw<__nv_bfloat16>& r) {
  r.u[0] = make_uint4(pack_bf16(x[0].x, x[0].y), pack_bf16(x[1].x, x[1].y), pack_bf16(x[2].x, x[2].y), pack_bf16(x[3].x, x[3].y));
}
__device__ __forceinline__ void load_pairs(const float* s, float2 (&x)[4]) {   // eight floats from shared memory
  const float4 a = reinterpret_cast<const float4*>(s)[0], b = reinterpret_cast<const float4*>(s)[1];
  x[0] = make_float2(a.x, a.y); x[1] = make_float2(a.z, a.w); x[2] = make_float2(b.x, b.y); x[3] = make_float2(b.z, b.w);
}

struct AppendArgs {
  const void *q, *k, *v, *q_norm, *k_norm;
  int64_t q_stride, k_stride, v_stride;
  const double* freq;
  void *pool, *q_out;                      // pool: of the layer
  int32_t* dev_status;
  float eps;
  int rot, H, per;                         // H: 0 without queries; per: heads of a unit
};

// A unit is `per` heads (a multiple of kHeads) of one token, of its H query, G key and G value heads; a warp takes it.
template <typename T>
__global__ void __launch_bounds__(kThreads, kCtas<T>) paged_append_kernel(Paged p, AppendArgs a) {
  constexpr int kUnroll = sizeof(T) == 2 ? 4 : 1;     // steps in flight
  __shared__ unsigned long long turn[kHeadDim / 2];   // freq / 2 pi modulo 1, times 2^64
  __shared__ __align__(16) float weight[2][kHeadDim];
  __shared__ __align__(16) float angle[kWarps][2][kHeadDim / 2];   // a warp's token: cosines, sines
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, sub = lane & 7;
  pdl_trigger();
  pdl_wait();
  const T *nq = static_cast<const T*>(a.q_norm), *nk = static_cast<const T*>(a.k_norm);
  if (tid < a.rot / 2) {
    const double t = a.freq[tid] * 0.15915494309189535;   // 1 / 2 pi
    turn[tid] = __double2ull_rn((t - floor(t)) * 18446744073709551616.0);
  }
  if (const T* w = tid < kHeadDim ? nq : nk) weight[tid / kHeadDim][tid % kHeadDim] = to_f<T>(w[tid % kHeadDim]);
  __syncthreads();
  const int rows = a.H + 2 * p.G, chunks = (rows + a.per - 1) / a.per, h8 = a.rot / 16;
  const int64_t units = (int64_t)p.T * chunks;
  // this lane's two groups of eight elements: a group of first members and its partners, or two groups that stay
  const bool turns = sub < h8;
  const int e0 = 8 * (turns ? sub : 2 * sub), e1 = 8 * (turns ? sub + h8 : 2 * sub + 1);
  T* pool = static_cast<T*>(a.pool);

  for (int64_t u = (int64_t)blockIdx.x * kWarps + warp; u < units; u += (int64_t)gridDim.x * kWarps) {
    const int t = (int)(u / chunks), lo = (int)(u % chunks) * a.per, hi = min(lo + a.per, rows);
    const T* q = static_cast<const T*>(a.q) + t * a.q_stride;
    const T* k = static_cast<const T*>(a.k) + t * a.k_stride - (int64_t)a.H * kHeadDim;
    const T* v = static_cast<const T*>(a.v) + t * a.v_stride - (int64_t)(a.H + p.G) * kHeadDim;
    float2 c[4], sn[4];                               // cosine and sine for this lane's pairs
    int s = 0, pos = 0, page = -1;
    bool placed = false;                              // the row's sequence and position are known
    for (int r0 = lo; r0 < hi; r0 += kHeads * kUnroll) {
      Raw<T> x0[kUnroll], x1[kUnroll];
#pragma unroll
      for (int i = 0; i < kUnroll; ++i) {
        const int row = r0 + kHeads * i + (lane >> 3);
        if (row >= hi) continue;
        const T* src = (row < a.H ? q : row < a.H + p.G ? k : v) + row * kHeadDim;
        x0[i] = load_raw(src + e0);
        x1[i] = load_raw(src + e1);
      }
      if (!placed) {                                  // behind the first loads
        s = count_le(p.row_start, p.S + 1, t, lane) - 1;
        if (s < 0 || s >= p.S) break;                 // a row of no sequence
        SeqRange r;
        if (!seq_range(p, s, r) || t < r.row0 || t >= r.row0 + r.n) {
          raise_status(a.dev_status, VARRATE_ERR_CORRUPT);
          break;
        }
        pos = r.len - r.n + (t - r.row0);
        page = __ldg(p.table + (int64_t)s * p.max_pages + (pos >> p.page_log2));
        if (page < 0 || page >= p.n_pages) {
          page = -1;
          raise_status(a.dev_status, VARRATE_ERR_CORRUPT);
        }
        if (a.rot) {
          __syncwarp();
#pragma unroll
          for (int i = lane; i < kHeadDim / 2; i += 32)
            if (i < a.rot / 2)
              sincospif(__ll2float_rn((long long)(turn[i] * (unsigned long long)pos)) * 0x1p-63f, &angle[warp][1][i], &angle[warp][0][i]);
          __syncwarp();
          if (turns) {
            load_pairs(angle[warp][0] + e0, c);
            load_pairs(angle[warp][1] + e0, sn);
          }
        }
        placed = true;
      }
#pragma unroll
      for (int i = 0; i < kUnroll; ++i) {
        const int row = r0 + kHeads * i + (lane >> 3);
        const bool is_q = row < a.H, is_v = row >= a.H + p.G;
        const bool normed = is_q ? nq != nullptr : nk != nullptr && !is_v;
        if ((nq || nk || a.rot) && r0 + kHeads * i < a.H + p.G) {   // else the warp's heads are copies
          float2 y0[4], y1[4];
          unpack(x0[i], y0);
          unpack(x1[i], y1);
          if (nq || nk) {
            float2 sq = make_float2(0.f, 0.f);
#pragma unroll
            for (int j = 0; j < 4; ++j) sq = fma2(y0[j], y0[j], fma2(y1[j], y1[j], sq));
            float ss = sq.x + sq.y;
#pragma unroll
            for (int o = 4; o > 0; o >>= 1) ss += __shfl_xor_sync(0xffffffffu, ss, o);
            if (normed) {
              const float f1 = rsqrtf(ss * (1.f / kHeadDim) + a.eps);
              const float2 f = make_float2(f1, f1);
              float2 w0[4], w1[4];
              load_pairs(weight[is_q ? 0 : 1] + e0, w0);
              load_pairs(weight[is_q ? 0 : 1] + e1, w1);
#pragma unroll
              for (int j = 0; j < 4; ++j) { y0[j] = mul2(mul2(y0[j], f), w0[j]); y1[j] = mul2(mul2(y1[j], f), w1[j]); }
            }
          }
          if (turns) {
#pragma unroll
            for (int j = 0; j < 4; ++j) {
              const float2 z = fma2(make_float2(-y1[j].x, -y1[j].y), sn[j], mul2(y0[j], c[j]));
              y1[j] = fma2(y0[j], sn[j], mul2(y1[j], c[j]));
              y0[j] = z;
            }
          }
          if (!is_v && (normed || turns)) { pack(y0, x0[i]); pack(y1, x1[i]); }
        }
        if (row >= hi || (!is_q && page < 0)) continue;
        T* dst = is_q ? static_cast<T*>(a.q_out) + ((int64_t)t * a.H + row) * kHeadDim
                      : pool + page_row(p, page, is_v, row - a.H - (is_v ? p.G : 0), pos & ((1 << p.page_log2) - 1)) * kHeadDim;
        store_raw(dst + e0, x0[i]);
        store_raw(dst + e1, x1[i]);
      }
    }
  }
  // every sequence's tables are checked, rows or not
  for (int s = blockIdx.x * kThreads + tid; s < p.S; s += gridDim.x * kThreads) {
    SeqRange r;
    if (!seq_range(p, s, r)) raise_status(a.dev_status, VARRATE_ERR_CORRUPT);
  }
}

template <typename T>
int launch(const Paged& p, AppendArgs& a, int layer, int num_sms, cudaStream_t st) {
  const int rows = a.H + 2 * p.G;
  // whole tokens per warp where there are enough of them, else their heads over several warps
  a.per = (rows + kHeads - 1) / kHeads * kHeads;
  while (a.per > kHeads && (int64_t)p.T * ((rows + a.per - 1) / a.per) < (int64_t)num_sms * kWarps * 4)
    a.per = (a.per / 2 + kHeads - 1) / kHeads * kHeads;
  a.pool = reinterpret_cast<T*>(p.pool) + (int64_t)layer * p.layer_rows * kHeadDim;
  const int64_t ctas = ((int64_t)p.T * ((rows + a.per - 1) / a.per) + kWarps - 1) / kWarps, most = (int64_t)num_sms * kCtas<T>;
  return launch_pdl(paged_append_kernel<T>, dim3((unsigned)(ctas < most ? ctas : most)), kThreads, 0, st, p, a) ? 1 : -1;
}

}  // namespace

int launch_paged_append(const Paged& p, int layer, int group, const void* q, int64_t q_stride, const void* k,
                        int64_t k_stride, const void* v, int64_t v_stride, const void* q_norm, const void* k_norm,
                        float eps, const double* freq, int rot, void* q_out, int32_t* dev_status, int num_sms,
                        cudaStream_t st) {
  AppendArgs a;
  a.q = q; a.k = k; a.v = v; a.q_norm = q ? q_norm : nullptr; a.k_norm = k_norm;
  a.q_stride = q_stride; a.k_stride = k_stride; a.v_stride = v_stride;
  a.freq = freq; a.q_out = q_out; a.dev_status = dev_status; a.eps = eps; a.rot = rot; a.H = q ? group * p.G : 0;
  return p.dtype == VARRATE_F32 ? launch<float>(p, a, layer, num_sms, st) : launch<__nv_bfloat16>(p, a, layer, num_sms, st);
}

}  // namespace vr
