// Paged cache, gather: a range of tokens of every sequence out of the pages into dense K and V.
//
// A copy: 16 threads (bf16) or 32 (fp32) move one token's row of a head, sixteen bytes each. A CTA takes kTokens tokens
// of one (sequence, layer, K or V, head) at a time, four rows in flight per thread. Bound by memory: four layers of 32768
// tokens, 8 heads, bf16: 174 us, 6.2 TB/s (91 % of a copy); 160 tokens of eight sequences: 4.3 us in a
// captured run, a launch.
#include "common.cuh"
#include "paged.h"

namespace vr {

namespace {

constexpr int kThreads = 256;
constexpr int kUnroll = 4;

template <int kRowBytes>
__global__ void __launch_bounds__(kThreads)
paged_gather_kernel(Paged p, int layer0, int n_layers, const int32_t* __restrict__ first, int n, uint4* __restrict__ k_out,
                    uint4* __restrict__ v_out, int32_t* dev_status, int64_t units, int chunks) {
  constexpr int kPer = kRowBytes / 16;                    // threads (16-byte pieces) of a row
  constexpr int kRows = kThreads / kPer, kTokens = kRows * kUnroll;
  const int tid = threadIdx.x, piece = tid % kPer, row = tid / kPer;
  const uint4* pool = reinterpret_cast<const uint4*>(p.pool);
  pdl_trigger();
  pdl_wait();
  for (int64_t u = blockIdx.x; u < units; u += gridDim.x) {
    // (sequence, layer, K or V, head, chunk), the chunk fastest
    int64_t x = u / chunks;
    const int chunk = (int)(u % chunks);
    const int g = (int)(x % p.G);
    x /= p.G;
    const int c = (int)(x & 1);
    x >>= 1;
    const int l = (int)(x % n_layers), s = (int)(x / n_layers);
    uint4* out = c ? v_out : k_out;
    if (out == nullptr) continue;
    const int f = first ? __ldg(first + s) : 0, len = __ldg(p.kv_len + s);
    if (f < 0 || (int64_t)f + n > len || len > kMaxLen || len > ((int64_t)p.max_pages << p.page_log2)) {
      if (tid == 0 && chunk == 0) raise_status(dev_status, VARRATE_ERR_CORRUPT);
      continue;
    }
    const int t0 = chunk * kTokens;                       // n is below a length now
    out += ((((int64_t)s * n_layers + l) * p.G + g) * n) * kPer + piece;
    const uint4* src = pool + (int64_t)(layer0 + l) * p.layer_rows * kPer + piece;
    int64_t from[kUnroll];
    uint4 val[kUnroll];
#pragma unroll
    for (int i = 0; i < kUnroll; ++i) {
      const int t = t0 + i * kRows + row, pos = f + t;
      from[i] = -1;
      if (t < n) {
        const int page = __ldg(p.table + (int64_t)s * p.max_pages + (pos >> p.page_log2));
        if (page >= 0 && page < p.n_pages) from[i] = page_row(p, page, c, g, pos & ((1 << p.page_log2) - 1)) * kPer;
        else raise_status(dev_status, VARRATE_ERR_CORRUPT);
      }
    }
#pragma unroll
    for (int i = 0; i < kUnroll; ++i)
      if (from[i] >= 0) val[i] = __ldcs(src + from[i]);
#pragma unroll
    for (int i = 0; i < kUnroll; ++i)
      if (from[i] >= 0) __stcs(out + (int64_t)(t0 + i * kRows + row) * kPer, val[i]);
  }
}

}  // namespace

int launch_paged_gather(const Paged& p, int layer, int n_layers, const int32_t* first, int n, void* k_out, void* v_out,
                        int32_t* dev_status, int num_sms, cudaStream_t st) {
  const int tokens = kThreads / (p.dtype == VARRATE_F32 ? 32 : 16) * kUnroll;
  const int chunks = n > kMaxLen ? 1 : (n + tokens - 1) / tokens;   // no sequence has more than kMaxLen
  const int64_t units = (int64_t)p.S * n_layers * 2 * p.G * chunks;
  const int grid = (int)(units < (int64_t)num_sms * 8 ? units : (int64_t)num_sms * 8);
  return launch_pdl(p.dtype == VARRATE_F32 ? paged_gather_kernel<512> : paged_gather_kernel<256>, dim3(grid), kThreads, 0, st,
                    p, layer, n_layers, first, n, (uint4*)k_out, (uint4*)v_out, dev_status, units, chunks)
             ? 1 : -1;
}

}  // namespace vr
