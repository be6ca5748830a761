// Paged cache in 8 bits: fragments of mma.sync products straight from the codes (internal).
#pragma once

#include "common.cuh"
#include "decode_common.cuh"
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

// Eight rows of queries as the B operand: lane (row g, t) has the elements 32 t .. 32 t + 31. fp16 times
// 2^n, the row's largest in [2^14, 2^15).
struct QueryFrags {
  uint32_t b[8][2];
  float f0, f1;            // for rows 2 t, 2 t + 1: what a product with them is multiplied by, 2^-n scale_log2

  __device__ __forceinline__ void load(const __nv_bfloat16* row, bool live, float scale_log2, int lane) {
    const int t = lane & 3;
    uint4 u[4];
#pragma unroll
    for (int i = 0; i < 4; ++i)
      u[i] = live ? __ldg(reinterpret_cast<const uint4*>(row + 32 * t + 8 * i)) : make_uint4(0, 0, 0, 0);
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

// Tiles of 16 tokens in shared memory: rows of 128 bytes, 16-byte pieces exchanged by the 128-byte swizzle, so that these reads meet
// no bank twice. tile: 1024-byte aligned.
__device__ __forceinline__ void read_keys(const unsigned char* tile, int lane, uint4 (&k)[4]) {
  const int g = lane >> 2, t = lane & 3;
#pragma unroll
  for (int i = 0; i < 4; ++i)
    k[i] = *reinterpret_cast<const uint4*>(tile + (g + 8 * (i >> 1)) * 128 + (((2 * t + (i & 1)) ^ g) << 4));
}
// Elements 16 g .. 16 g + 15 of keys 2 t, 2 t + 1, 2 t + 8, 2 t + 9.
__device__ __forceinline__ void read_values(const unsigned char* tile, int lane, uint4 (&v)[4]) {
  const int g = lane >> 2, t = lane & 3;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const int key = 2 * t + (i & 1);
    v[i] = *reinterpret_cast<const uint4*>(tile + (key + 8 * (i >> 1)) * 128 + ((g ^ key) << 4));
  }
}

// A warp's steps of 16 keys: first, first + stride, ..., n of them, of one sequence and KV head. Pages and scale bytes are
// fetched for 32 steps at a time, a lane each, one batch ahead.
struct Steps {
  const Paged& p;
  const unsigned char* scale;
  const int32_t* table;
  int32_t* dev_status;
  int g, first, stride, n, batch;
  int page0, page1;
  uint32_t bytes0, bytes1;   // of the key's block, and times 256 of the value's

  __device__ __forceinline__ int in_page(int i) const { return ((first + i * stride) << 4) & ((1 << p.page_log2) - 1); }
  __device__ __forceinline__ int row(int page, int i) const { return (int)page_row(p, max(page, 0), 0, g, in_page(i)); }
  __device__ __forceinline__ void fetch(int b, int lane, int& page, uint32_t& bytes) {
    const int i = 32 * b + lane;
    page = 0;
    bytes = 0;
    if (i >= n) return;
    page = __ldg(table + (((first + i * stride) << 4) >> p.page_log2));
    if (page < 0 || page >= p.n_pages) { raise_status(dev_status, VARRATE_ERR_CORRUPT); page = -1; }
    const int r = row(page, i);
    bytes = __ldg(scale + scale_at(r)) | (uint32_t)__ldg(scale + scale_at(r + (p.G << p.page_log2))) << 8;
  }
  __device__ __forceinline__ void start(int lane) {
    batch = 0;
    fetch(0, lane, page0, bytes0);
    fetch(1, lane, page1, bytes1);
  }
  // of step i, of the current batch or the next one; a page out of range is -1 (its row is one of page 0)
  __device__ __forceinline__ int page(int i) const { return __shfl_sync(0xffffffffu, (i >> 5) == batch ? page0 : page1, i & 31); }
  __device__ __forceinline__ uint32_t bytes(int i) const { return __shfl_sync(0xffffffffu, (i >> 5) == batch ? bytes0 : bytes1, i & 31); }
  __device__ __forceinline__ void done(int i, int lane) {   // with step i
    if ((i & 31) != 31) return;
    page0 = page1;
    bytes0 = bytes1;
    fetch(++batch + 1, lane, page1, bytes1);
  }
};

// Sequences of at most this many new tokens are taken by mma.sync: one or two blocks of eight rows; more by tcgen05, whose kernel is
// launched where a sequence can have more (which ones do is known on the device only) and ends at once where none does. A batch of as many
// rows as sequences is taken for one of single tokens, all for mma.sync: 64 on 1000 tokens take 38.7 us with that kernel alone, 45.4
// with the other one launched as well. One with fewer rows than sequences has empty slots, and may have a chunk beside them: 60 tokens on
// 32768 and 63 empty slots take 297 us by mma.sync and 48 by tcgen05 (weights 268 and 37), 8 tokens 48 and 42, so up to four blocks of
// rows the one kernel does.
inline int few_tokens(const Paged& p, int group) {
  const int block = 8 / group;
  return p.T == p.S || (p.T < p.S && p.T <= 4 * block) ? p.T : 2 * block;
}

__device__ __forceinline__ bool warp_wait(uint64_t* bar, uint32_t parity) {
  for (uint32_t i = 0; i < kWaitTries; ++i)
    if (__all_sync(0xffffffffu, mbar_try_wait(bar, parity))) return true;
  return false;
}

// Products of 16 keys with the rows: keys[2 i + h] is the 16 bytes at element 32 t + 16 h of key g + 8 i. Out: (key g, row 2 t),
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
