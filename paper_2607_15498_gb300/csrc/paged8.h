// Paged cache in 8 bits: what its append, attention, weight and eviction kernels share (internal; the public ABI is
// include/varrate.h).
#pragma once

#include <cuda_runtime.h>
#include <stddef.h>
#include <stdint.h>

#include "common.cuh"
#include "paged.h"

namespace vr {

constexpr int kBlock = 16, kBlockLog2 = 4;   // tokens that share a scale

// The pages of one call, and its batch: p.pool holds the codes, a row of 128 bytes a token, head, K or V.
struct Paged8 {
  Paged p;
  unsigned char* scale;    // [layer][row / 16] by the rows of the codes
  float* mass;             // [layer][page][G][page_size], or null
};

// Scale byte of the block that holds a row of the codes (page_row).
__host__ __device__ __forceinline__ int64_t scale_at(int64_t row) { return row >> kBlockLog2; }
// Token `in_page` of page `page`, head g, of one layer's weights.
__host__ __device__ __forceinline__ int64_t mass_at(const Paged& p, int page, int g, int in_page) {
  return (((int64_t)page * p.G + g) << p.page_log2) + in_page;
}

// Scale bytes: byte b stands for 2^(b - 127); 0 for a block of zeros.
constexpr int kMaxScale = 246;               // 448 * 2^119 is the last that bf16 holds as well
// Least byte whose scale times 448 is not below amax (finite, >= 0): 448 = 1.75 * 2^8, so the exponent of amax less 8, one
// more where its mantissa is above 1.75.
__device__ __forceinline__ int scale_byte(float amax) {
  if (amax == 0.f) return 0;
  const int b = (int)((__float_as_uint(amax) + 0x1fffffu) >> 23) - 8;
  return min(max(b, 1), kMaxScale);
}
// 1 / scale
__device__ __forceinline__ float scale_inverse(int byte) { return __uint_as_float((uint32_t)(254 - byte) << 23); }

// Two numbers as e4m3 codes (lo in the low byte), to the nearest, ties to even; past 448 they are 448, NaN stays NaN.
__device__ __forceinline__ uint32_t codes2(float lo, float hi) {
  uint16_t r;
  asm("cvt.rn.satfinite.e4m3x2.f32 %0, %1, %2;\n" : "=h"(r) : "f"(hi), "f"(lo));
  return r;
}
// Codes of a block whose scale grows by 2^k, k >= 0: exact but for numbers below 2^-6 of the new scale, which lose places. In
// fp16 every product that does not round to zero is exact.
struct Rescale {
  __half2 f;
  __device__ __forceinline__ explicit Rescale(int k) {
    k = min(k, 24);
    f = __half2half2(__ushort_as_half((unsigned short)(k < 15 ? (15 - k) << 10 : 1 << (24 - k))));
  }
  __device__ __forceinline__ uint32_t two(uint32_t w) const {
    uint32_t h;
    uint16_t r;
    asm("cvt.rn.f16x2.e4m3x2 %0, %1;\n" : "=r"(h) : "h"((uint16_t)w));
    const __half2 y = __hmul2(reinterpret_cast<const __half2&>(h), f);
    asm("cvt.rn.satfinite.e4m3x2.f16x2 %0, %1;\n" : "=h"(r) : "r"(reinterpret_cast<const uint32_t&>(y)));
    return r;
  }
  __device__ __forceinline__ uint32_t four(uint32_t w) const { return two(w & 0xffffu) | two(w >> 16) << 16; }
};

int launch_paged8_append(const Paged8& c, int layer, int group, const void* q, int64_t q_stride, const void* k,
                         int64_t k_stride, const void* v, int64_t v_stride, const void* q_norm, const void* k_norm,
                         float eps, const double* freq, int rot, const int32_t* gone, void* q_out, int32_t* dev_status,
                         int num_sms, cudaStream_t st);
size_t paged8_attn_ws_bytes(const Paged8& c, int group, int num_sms);
int launch_paged8_attn(const Paged8& c, int layer, int group, const void* q, void* out, float* lse, int32_t* dev_status,
                       void* ws, int num_sms, cudaStream_t st);
// The sequences of n_min new tokens and more, on tcgen05: the second header of workspace `ws`, partials to `part`, not merged.
int launch_paged8_attn_tc(const Paged8& c, int layer, int group, int n_min, const void* q, void* out, float* lse,
                          int32_t* dev_status, void* ws, float* part, int num_sms, cudaStream_t st);
// Merges the partials of both, and writes lse of the rows that were cut: the first kernel took the sequences of at most `few`
// new tokens, with tq tokens a block; the second the others, with partials from `second` on (null: not launched) and blocks of 2 tq2.
struct Merge8 {
  float* second;
  float* lse;               // [T][H], or null
  int few, tq2;
};
int launch_paged8_merge(const Paged& p, int group, void* out, int32_t* dev_status, void* ws, int tq, const Merge8& two,
                        int num_sms, cudaStream_t st);
int launch_paged8_mass(const Paged8& c, int layer, int group, const void* q, const float* lse, int32_t* dev_status,
                       int num_sms, cudaStream_t st);
// The sequences of more than few_tokens(group) new tokens, on tcgen05.
int launch_paged8_mass_tc(const Paged8& c, int layer, int group, const void* q, const float* lse, int32_t* dev_status,
                          int num_sms, cudaStream_t st);
int launch_paged8_evict(const Paged8& c, int layer, int n_layers, int budget, int n_first, int n_last, int32_t* kept,
                        int32_t* new_len, int32_t* gone, int32_t* dev_status, int num_sms, cudaStream_t st);

}  // namespace vr
