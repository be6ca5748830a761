// Paged cache, attention of new tokens over the pages: causal softmax attention, one pass over the keys and values
// with the running maximum and sum of every row.
//
// The rows of a CTA are kRows (token, query head) pairs of one KV head, so a key read once serves the whole group.
// Scores of 32 keys at a time, four rows and two keys a thread; weights through shared memory to the values, four
// rows and eight columns a thread. All arithmetic in fp32.
#include <math.h>

#include "common.cuh"
#include "paged.h"

namespace vr {

namespace {

constexpr int kThreads = 256;
constexpr int kRows = 64, kKeys = 32;
constexpr int kPitch = kHeadDim + 4;       // floats of a query or key row: 16-byte reads of 8 rows fall on 32 banks
constexpr int kPPitch = kKeys + 4;

struct Smem {
  float q[kRows][kPitch];
  float k[kKeys][kPitch];
  float v[kKeys][kHeadDim];
  float p[kRows][kPPitch];
  int seq, block;
};

__device__ __forceinline__ void set4(float* d, float4 x) { *reinterpret_cast<float4*>(d) = x; }
__device__ __forceinline__ float4 get4(const float* s) { return *reinterpret_cast<const float4*>(s); }

template <typename T>
__global__ void __launch_bounds__(kThreads)
paged_attn_kernel(Paged p, const T* __restrict__ pool, const T* __restrict__ q, T* __restrict__ out, int32_t* dev_status,
                  int grp, float scale) {
  extern __shared__ __align__(16) unsigned char raw[];
  Smem& sm = *reinterpret_cast<Smem*>(raw);
  const int tid = threadIdx.x, lane = tid & 31, g = blockIdx.y, H = p.G * grp;
  const int tq = kRows / grp;               // tokens of a CTA
  if (tid < 32) {                           // which (sequence, block) this CTA has: blocks of all sequences in order
    int before = 0, seq = -1, block = 0;
    for (int s0 = 0; s0 < p.S && seq < 0; s0 += 32) {
      int nb = 0;
      if (s0 + lane < p.S) {
        SeqRange r;
        if (seq_range(p, s0 + lane, r)) nb = (r.n + tq - 1) / tq;
        else raise_status(dev_status, VARRATE_ERR_CORRUPT);
      }
      int incl = nb;
#pragma unroll
      for (int o = 1; o < 32; o <<= 1) {
        const int y = __shfl_up_sync(0xffffffffu, incl, o);
        if (lane >= o) incl += y;
      }
      const int at = (int)blockIdx.x - before;
      const unsigned hit = __ballot_sync(0xffffffffu, at >= incl - nb && at < incl);
      if (hit) {
        const int l = __ffs(hit) - 1;
        seq = s0 + l;
        block = __shfl_sync(0xffffffffu, nb - 1 - (at - (incl - nb)), l);   // the longest first
      }
      before += __shfl_sync(0xffffffffu, incl, 31);
    }
    if (lane == 0) { sm.seq = seq; sm.block = block; }
  }
  __syncthreads();
  if (sm.seq < 0) return;
  SeqRange r;
  seq_range(p, sm.seq, r);
  const int t0 = sm.block * tq, nt = min(tq, r.n - t0), rows = nt * grp;
  const int pos0 = r.len - r.n + t0;        // position of the first row's token
  const int end = pos0 + nt;                // keys that any row sees
  const int32_t* table = p.table + (int64_t)sm.seq * p.max_pages;
  const T* qb = q + ((int64_t)(r.row0 + t0) * H + (int64_t)g * grp) * kHeadDim;
  for (int i = tid; i < kRows * 32; i += kThreads) {
    const int row = i >> 5, c = (i & 31) * 4;
    float4 x = make_float4(0.f, 0.f, 0.f, 0.f);
    if (row < rows) x = load4(qb + ((int64_t)(row / grp) * H + row % grp) * kHeadDim + c);
    set4(&sm.q[row][c], make_float4(x.x * scale, x.y * scale, x.z * scale, x.w * scale));
  }
  const int ty = tid >> 4, tx = tid & 15;
  int sees[4];                              // keys that the thread's rows see
#pragma unroll
  for (int i = 0; i < 4; ++i) sees[i] = min(pos0 + (4 * ty + i) / grp + 1, end);
  float m[4], l[4], o[4][8];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    m[i] = -INFINITY;
    l[i] = 0.f;
#pragma unroll
    for (int j = 0; j < 8; ++j) o[i][j] = 0.f;
  }
  for (int k0 = 0; k0 < end; k0 += kKeys) {
    __syncthreads();
    for (int i = tid; i < 2 * kKeys * 32; i += kThreads) {
      const int c = i >> 10, key = (i >> 5) & 31, col = (i & 31) * 4, u = k0 + key;
      float4 x = make_float4(0.f, 0.f, 0.f, 0.f);
      if (u < end) {
        const int page = __ldg(table + (u >> p.page_log2));
        if (page >= 0 && page < p.n_pages)
          x = load4(pool + page_row(p, page, c, g, u & ((1 << p.page_log2) - 1)) * kHeadDim + col);
        else raise_status(dev_status, VARRATE_ERR_CORRUPT);
      }
      set4(c ? &sm.v[key][col] : &sm.k[key][col], x);
    }
    __syncthreads();
    float s[4][2] = {};
#pragma unroll 8
    for (int d = 0; d < kHeadDim; d += 4) {
      float4 a[4], b[2];
#pragma unroll
      for (int i = 0; i < 4; ++i) a[i] = get4(&sm.q[4 * ty + i][d]);
#pragma unroll
      for (int j = 0; j < 2; ++j) b[j] = get4(&sm.k[tx + 16 * j][d]);
#pragma unroll
      for (int i = 0; i < 4; ++i)
#pragma unroll
        for (int j = 0; j < 2; ++j)
          s[i][j] = fmaf(a[i].x, b[j].x, fmaf(a[i].y, b[j].y, fmaf(a[i].z, b[j].z, fmaf(a[i].w, b[j].w, s[i][j]))));
    }
#pragma unroll
    for (int i = 0; i < 4; ++i) {
#pragma unroll
      for (int j = 0; j < 2; ++j)
        if (k0 + tx + 16 * j >= sees[i]) s[i][j] = -INFINITY;
      float mx = fmaxf(s[i][0], s[i][1]);
#pragma unroll
      for (int w = 8; w > 0; w >>= 1) mx = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, w));
      const float mn = fmaxf(m[i], mx), ref = mn == -INFINITY ? 0.f : mn;   // no finite score yet: weights 0
      const float f = exp2f((m[i] - ref) * kLog2e);
      m[i] = mn;
      float sum = 0.f;
#pragma unroll
      for (int j = 0; j < 2; ++j) {
        const float w = exp2f((s[i][j] - ref) * kLog2e);
        sm.p[4 * ty + i][tx + 16 * j] = w;
        sum += w;
      }
      l[i] = l[i] * f + sum;
#pragma unroll
      for (int j = 0; j < 8; ++j) o[i][j] *= f;
    }
    __syncthreads();
    const bool partial = k0 + kKeys > pos0 + 1;   // some row does not see all of these keys: weight 0 is no product there
#pragma unroll 2
    for (int key = 0; key < kKeys; key += 4) {
      float w[4][4];
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const float4 x = get4(&sm.p[4 * ty + i][key]);
        w[i][0] = x.x; w[i][1] = x.y; w[i][2] = x.z; w[i][3] = x.w;
      }
#pragma unroll
      for (int kk = 0; kk < 4; ++kk) {
        const float4 v0 = get4(&sm.v[key + kk][4 * tx]), v1 = get4(&sm.v[key + kk][64 + 4 * tx]);
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          if (partial && k0 + key + kk >= sees[i]) continue;
          const float a = w[i][kk];
          o[i][0] = fmaf(a, v0.x, o[i][0]); o[i][1] = fmaf(a, v0.y, o[i][1]);
          o[i][2] = fmaf(a, v0.z, o[i][2]); o[i][3] = fmaf(a, v0.w, o[i][3]);
          o[i][4] = fmaf(a, v1.x, o[i][4]); o[i][5] = fmaf(a, v1.y, o[i][5]);
          o[i][6] = fmaf(a, v1.z, o[i][6]); o[i][7] = fmaf(a, v1.w, o[i][7]);
        }
      }
    }
  }
  T* ob = out + ((int64_t)(r.row0 + t0) * H + (int64_t)g * grp) * kHeadDim;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const int row = 4 * ty + i;
    float sum = l[i];
#pragma unroll
    for (int w = 8; w > 0; w >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, w);
    if (row >= rows) continue;
    const float f = sum == 0.f ? 0.f : 1.f / sum;
    T* d = ob + ((int64_t)(row / grp) * H + row % grp) * kHeadDim;
#pragma unroll
    for (int j = 0; j < 8; ++j) d[(j >> 2) * 64 + 4 * tx + (j & 3)] = from_f<T>(o[i][j] * f);
  }
}

template <typename T>
int launch(const Paged& p, int layer, int group, const void* q, void* out, int32_t* dev_status, cudaStream_t st) {
  const int tq = kRows / group;
  const int64_t blocks = p.T / tq + (p.S < p.T ? p.S : p.T);   // at least one more than full blocks per sequence
  if (cudaFuncSetAttribute(paged_attn_kernel<T>, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)sizeof(Smem)) != cudaSuccess)
    return -1;
  const T* pool = reinterpret_cast<const T*>(p.pool) + (int64_t)layer * p.layer_rows * kHeadDim;
  paged_attn_kernel<T><<<dim3((unsigned)blocks, p.G), kThreads, sizeof(Smem), st>>>(
      p, pool, (const T*)q, (T*)out, dev_status, group, 1.f / sqrtf((float)kHeadDim));
  return 1;
}

}  // namespace

size_t paged_attn_ws_bytes(const Paged& p, int group, int num_sms) {
  return p.dtype == VARRATE_F32 ? 256 : paged_attn_tc_ws_bytes(p, group, num_sms);
}

int launch_paged_attn(const Paged& p, int layer, int group, const void* q, void* out, int32_t* dev_status, void* ws,
                      int num_sms, cudaStream_t st) {
  return p.dtype == VARRATE_F32 ? launch<float>(p, layer, group, q, out, dev_status, st)
                                : launch_paged_attn_tc(p, layer, group, q, out, dev_status, ws, num_sms, st);
}

}  // namespace vr
