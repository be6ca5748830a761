// Paged cache: what the append, attention and gather kernels share (internal; the public ABI is include/varrate.h).
#pragma once

#include <cuda_runtime.h>
#include <stddef.h>
#include <stdint.h>

#include "common.cuh"

namespace vr {

// The pages of one call, and its batch (row_start is not used by gather).
struct Paged {
  unsigned char* pool;
  int64_t layer_rows;      // n_pages * 2 * G * page_size: rows of d elements in one layer
  int n_pages, G, page_log2, dtype;
  const int32_t* row_start;
  const int32_t* kv_len;
  const int32_t* table;
  int S, max_pages, T;
};

// Row of the pool (of d elements, in one layer) that holds token `in_page` of page `page`, head g, K (0) or V (1).
__host__ __device__ __forceinline__ int64_t page_row(const Paged& p, int page, int kv, int g, int in_page) {
  return ((((int64_t)page * 2 + kv) * p.G + g) << p.page_log2) + in_page;
}

constexpr int kMaxLen = 0x7fffff00;   // tokens of a sequence: positions a key tile further stay below 2^31

// What one sequence brings: its first row, its new tokens and all of its tokens; false where the tables
// are out of range (see varrate_seqs).
struct SeqRange {
  int row0, n, len;
};
__device__ __forceinline__ bool seq_range(const Paged& p, int s, SeqRange& r) {
  const int a = __ldg(p.row_start + s), b = __ldg(p.row_start + s + 1), len = __ldg(p.kv_len + s);
  r.row0 = a; r.n = b - a; r.len = len;
  return a >= 0 && b >= a && b <= p.T && len >= r.n && len <= kMaxLen && len <= ((int64_t)p.max_pages << p.page_log2);
}

// Entries of a[0 .. n) that are <= t, a sorted; one warp. (Unsorted: some number in [0, n].)
__device__ __forceinline__ int count_le(const int32_t* a, int n, int t, int lane) {
  int lo = 0;
  while (n > 32) {
    const int step = (n + 31) >> 5, i = (lane + 1) * step - 1;   // last entry of the lane's part
    const bool le = i < n && __ldg(a + lo + i) <= t;
    const int k = __popc(__ballot_sync(0xffffffffu, le));
    lo += k * step;
    n = min(step, n - k * step);
  }
  const bool le = lane < n && __ldg(a + lo + lane) <= t;
  return lo + __popc(__ballot_sync(0xffffffffu, le));
}

// Two floats in one instruction.
__device__ __forceinline__ float2 fma2(float2 a, float2 b, float2 c) {
  float2 d;
  asm("fma.rn.f32x2 %0, %1, %2, %3;\n" : "=l"(reinterpret_cast<uint64_t&>(d))
      : "l"(reinterpret_cast<uint64_t&>(a)), "l"(reinterpret_cast<uint64_t&>(b)), "l"(reinterpret_cast<uint64_t&>(c)));
  return d;
}
__device__ __forceinline__ float2 add2(float2 a, float2 b) {
  float2 d;
  asm("add.rn.f32x2 %0, %1, %2;\n" : "=l"(reinterpret_cast<uint64_t&>(d))
      : "l"(reinterpret_cast<uint64_t&>(a)), "l"(reinterpret_cast<uint64_t&>(b)));
  return d;
}
__device__ __forceinline__ float2 mul2(float2 a, float2 b) {
  float2 d;
  asm("mul.rn.f32x2 %0, %1, %2;\n" : "=l"(reinterpret_cast<uint64_t&>(d))
      : "l"(reinterpret_cast<uint64_t&>(a)), "l"(reinterpret_cast<uint64_t&>(b)));
  return d;
}

// Launch with programmatic stream serialization: the kernel waits (pdl_wait) before it touches memory.
template <typename... P, typename... A>
inline bool launch_pdl(void (*kernel)(P...), dim3 grid, int threads, size_t smem, cudaStream_t st, A... args) {
  cudaLaunchAttribute pdl[1];
  pdl[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  pdl[0].val.programmaticStreamSerializationAllowed = 1;
  cudaLaunchConfig_t lc = {};
  lc.gridDim = grid;
  lc.blockDim = dim3(threads);
  lc.dynamicSmemBytes = smem;
  lc.stream = st;
  lc.attrs = pdl;
  lc.numAttrs = 1;
  return cudaLaunchKernelEx(&lc, kernel, P(args)...) == cudaSuccess;
}

int launch_paged_append(const Paged& p, int layer, int group, const void* q, int64_t q_stride, const void* k,
                        int64_t k_stride, const void* v, int64_t v_stride, const void* q_norm, const void* k_norm,
                        float eps, const double* freq, int rot, void* q_out, int32_t* dev_status, int num_sms,
                        cudaStream_t st);
int launch_paged_gather(const Paged& p, int layer, int n_layers, const int32_t* first, int n, void* k_out, void* v_out,
                        int32_t* dev_status, int num_sms, cudaStream_t st);
size_t paged_attn_ws_bytes(const Paged& p, int group, int num_sms);
size_t paged_attn_tc_ws_bytes(const Paged& p, int group, int num_sms);
int launch_paged_attn_tc(const Paged& p, int layer, int group, const void* q, void* out, int32_t* dev_status, void* ws,
                         int num_sms, cudaStream_t st);
int launch_paged_attn(const Paged& p, int layer, int group, const void* q, void* out, int32_t* dev_status, void* ws,
                      int num_sms, cudaStream_t st);

}  // namespace vr
