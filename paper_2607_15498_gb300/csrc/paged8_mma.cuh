// Paged cache in 8 bits: fragments of mma.sync products straight from the codes (internal).
#pragma once

#include "common.cuh"
#include "paged8.h"

namespace vr {

__device__ __forceinline__ uint32_t pack_f16(float lo, float hi) {
  const __half2 v = __floats2half2_rn(lo, hi);
  return reinterpret_cast<const uint32_t&>(v);
}
// D(16x8, fp32) += A(16x16, fp16, row) * B(16x8, fp16, col)
__device__ __forceinline__ void mma_f16_16816(float (&d)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1) {
  asm("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, "
      "{%8,%9}, {%0,%1,%2,%3};\n"
      : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
      : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}
// Two codes (of the low 16 bits) as two fp16, or two bf16: exact both.
__device__ __forceinline__ uint32_t f16_codes(uint32_t w) {
  uint32_t h;
  asm("cvt.rn.f16x2.e4m3x2 %0, %1;\n" : "=r"(h) : "h"((uint16_t)w));
  return h;
}
__device__ __forceinline__ uint32_t bf16_codes(uint32_t w) {
  const uint32_t h = f16_codes(w);
  const float2 f = __half22float2(reinterpret_cast<const __half2&>(h));
  return pack_bf16(f.x, f.y);
}
// Elements 2 j and 2 j + 1 of a lane's 16 of two keys: (a, b) of the first in the low half, of the second in the high one.
__device__ __forceinline__ uint32_t value_bytes(const uint4& a, const uint4& b, int j) {
  const uint32_t wa = j < 2 ? a.x : j < 4 ? a.y : j < 6 ? a.z : a.w, wb = j < 2 ? b.x : j < 4 ? b.y : j < 6 ? b.z : b.w;
  return __byte_perm(wa, wb, j & 1 ? 0x7362 : 0x5140);
}

// Eight rows of queries as the B operand: lane (row g, t) has the elements 16 t .. 16 t + 15 and those 64 further. fp16 times
// 2^n, the row's largest in [2^14, 2^15).
struct QueryFrags {
  uint32_t b[8][2];
  float f0, f1;            // for rows 2 t, 2 t + 1: what a product with them is multiplied by, 2^-n scale_log2

  __device__ __forceinline__ void load(const __nv_bfloat16* row, bool live, float scale_log2, int lane) {
    const int t = lane & 3;
    uint4 u[4];
#pragma unroll
    for (int i = 0; i < 4; ++i)
      u[i] = live ? __ldg(reinterpret_cast<const uint4*>(row + 16 * t + 64 * (i >> 1) + 8 * (i & 1))) : make_uint4(0, 0, 0, 0);
    float top = 0.f;
#pragma unroll
    for (int i = 0; i < 16; ++i) {
      const uint32_t w = reinterpret_cast<const uint32_t*>(u)[i];
      const float a = fabsf(__uint_as_float(w << 16)), b = fabsf(__uint_as_float(w & 0xffff0000u));
      top = fmaxf(top, fmaxf(a < INFINITY ? a : 0.f, b < INFINITY ? b : 0.f));
    }
    top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, 1));
    top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, 2));
    const int n = top == 0.f ? 0 : min(126, 14 + 127 - (int)(__float_as_uint(top) >> 23));
    const float up = __uint_as_float((uint32_t)(127 + n) << 23);
#pragma unroll
    for (int i = 0; i < 16; ++i) {
      const uint32_t w = reinterpret_cast<const uint32_t*>(u)[i];
      b[i >> 1][i & 1] = pack_f16(__uint_as_float(w << 16) * up, __uint_as_float(w & 0xffff0000u) * up);
    }
    const float f = scale_log2 * __uint_as_float((uint32_t)max(127 - n, 1) << 23);
    f0 = __shfl_sync(0xffffffffu, f, 8 * t);
    f1 = __shfl_sync(0xffffffffu, f, 8 * t + 4);
  }
};

// Products of 16 keys with the rows: keys[2 i + h] is the 16 bytes at element 16 t + 64 h of key g + 8 i. Out: (key g, row 2 t),
// (g, 2 t + 1), (g + 8, 2 t), (g + 8, 2 t + 1).
__device__ __forceinline__ void key_scores(const uint4 (&keys)[4], const QueryFrags& q, float (&s)[4]) {
  float d[2][4] = {{0.f, 0.f, 0.f, 0.f}, {0.f, 0.f, 0.f, 0.f}};
#pragma unroll
  for (int h = 0; h < 2; ++h) {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const uint32_t lo = reinterpret_cast<const uint32_t*>(&keys[h])[i], hi = reinterpret_cast<const uint32_t*>(&keys[2 + h])[i];
      const uint32_t a[4] = {f16_codes(lo), f16_codes(hi), f16_codes(lo >> 16), f16_codes(hi >> 16)};
      mma_f16_16816(d[h], a, q.b[4 * h + i][0], q.b[4 * h + i][1]);
    }
  }
#pragma unroll
  for (int i = 0; i < 4; ++i) s[i] = d[0][i] + d[1][i];
}

}  // namespace vr
