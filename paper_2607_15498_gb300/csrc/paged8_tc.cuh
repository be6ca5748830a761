// Paged cache in 8 bits on tcgen05: what the attention and the weights share (internal).
#pragma once

#include "common.cuh"
#include "paged_tc.cuh"

namespace vr {

// Registers a thread of a warpgroup from here on. At the head of the branch that the warpgroup takes: elsewhere the compiler spills.
template <int kRegs> __device__ __forceinline__ void more_registers() { asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;\n" ::"n"(kRegs)); }
template <int kRegs> __device__ __forceinline__ void fewer_registers() { asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;\n" ::"n"(kRegs)); }
// Whether a kernel was compiled to as many registers a thread as its warpgroups share out in sum (a wait for more would not end).
template <typename F>
inline bool registers_for(F* kernel, int threads, int shared_out) {
  cudaFuncAttributes a;
  return cudaFuncGetAttributes(&a, kernel) == cudaSuccess && a.numRegs * threads >= shared_out;
}

// 32 columns on their way; they are there after the wait, which waits for all that the thread has asked for.
__device__ __forceinline__ void tmem_ld32_async(uint32_t taddr, float (&v)[32]) {
  asm volatile(
      "tcgen05.ld.sync.aligned.32x32b.x32.b32 {%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,"
      "%16,%17,%18,%19,%20,%21,%22,%23,%24,%25,%26,%27,%28,%29,%30,%31}, [%32];\n"
      : "=f"(v[0]), "=f"(v[1]), "=f"(v[2]), "=f"(v[3]), "=f"(v[4]), "=f"(v[5]), "=f"(v[6]), "=f"(v[7]), "=f"(v[8]),
        "=f"(v[9]), "=f"(v[10]), "=f"(v[11]), "=f"(v[12]), "=f"(v[13]), "=f"(v[14]), "=f"(v[15]), "=f"(v[16]),
        "=f"(v[17]), "=f"(v[18]), "=f"(v[19]), "=f"(v[20]), "=f"(v[21]), "=f"(v[22]), "=f"(v[23]), "=f"(v[24]),
        "=f"(v[25]), "=f"(v[26]), "=f"(v[27]), "=f"(v[28]), "=f"(v[29]), "=f"(v[30]), "=f"(v[31])
      : "r"(taddr) : "memory");
}
__device__ __forceinline__ void tmem_wait_ld32(float (&v)[32]) {
  asm volatile("tcgen05.wait::ld.sync.aligned;\n"
      : "+f"(v[0]), "+f"(v[1]), "+f"(v[2]), "+f"(v[3]), "+f"(v[4]), "+f"(v[5]), "+f"(v[6]), "+f"(v[7]), "+f"(v[8]),
        "+f"(v[9]), "+f"(v[10]), "+f"(v[11]), "+f"(v[12]), "+f"(v[13]), "+f"(v[14]), "+f"(v[15]), "+f"(v[16]),
        "+f"(v[17]), "+f"(v[18]), "+f"(v[19]), "+f"(v[20]), "+f"(v[21]), "+f"(v[22]), "+f"(v[23]), "+f"(v[24]),
        "+f"(v[25]), "+f"(v[26]), "+f"(v[27]), "+f"(v[28]), "+f"(v[29]), "+f"(v[30]), "+f"(v[31]) :: "memory");
}

// A lane's 16 codes as bf16 times the scale 2^(byte - 127): exact but for numbers below 2^-133.
__device__ __forceinline__ void expand16(const uint4& w, uint32_t scale2, uint4& lo, uint4& hi) {
  const uint32_t in[4] = {w.x, w.y, w.z, w.w};
  uint32_t r[8];
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    uint32_t h;
    asm("cvt.rn.f16x2.e4m3x2 %0, %1;\n" : "=r"(h) : "h"((uint16_t)(in[i >> 1] >> (16 * (i & 1)))));
    const float2 f = __half22float2(reinterpret_cast<const __half2&>(h));
    const uint32_t b = pack_bf16(f.x, f.y);
    asm("mul.rn.bf16x2 %0, %1, %2;\n" : "=r"(r[i]) : "r"(b), "r"(scale2));
  }
  lo = make_uint4(r[0], r[1], r[2], r[3]);
  hi = make_uint4(r[4], r[5], r[6], r[7]);
}

// Key `key` of a tile: its 128 codes as 128 bf16 times the scale 2^(byte - 127), or as fp16 without it; zeros where it is not
// `there`. The tile is two panels of `rows` rows of 64 elements, 128-byte swizzle; the codes stand, swizzled as well, where the second half
// of the key's row will be, and 16 of them are read before anything is written there, so a thread per key needs nobody. The
// loop is short, as the softmax beside it wants the instruction cache.
template <bool kScaled>
__device__ __forceinline__ void expand_row(unsigned char* tile, int rows, int key, bool there, uint32_t byte) {
  unsigned char *row = tile + key * 128, *codes = row + rows * 128;
  const uint32_t scale2 = byte * 0x00800080u;
  auto read = [&](int i) { return *reinterpret_cast<const uint4*>(codes + ((i ^ (key & 7)) << 4)); };
  uint4 next = read(0);
#pragma unroll 1
  for (int i = 0; i < 8; ++i) {                             // elements 16 i .. 16 i + 15
    uint4 w = next, lo, hi;
    next = read((i + 1) & 7);                               // (the last one is not used)
    if (!there) w = make_uint4(0, 0, 0, 0);
    if constexpr (kScaled) {
      expand16(w, scale2, lo, hi);
    } else {
      const uint32_t in[4] = {w.x, w.y, w.z, w.w};
      uint32_t r[8];
#pragma unroll
      for (int j = 0; j < 8; ++j) asm("cvt.rn.f16x2.e4m3x2 %0, %1;\n" : "=r"(r[j]) : "h"((uint16_t)(in[j >> 1] >> (16 * (j & 1)))));
      lo = make_uint4(r[0], r[1], r[2], r[3]);
      hi = make_uint4(r[4], r[5], r[6], r[7]);
    }
    unsigned char* at = i < 4 ? row : codes;
    const int piece = 2 * (i & 3);
    *reinterpret_cast<uint4*>(at + ((piece ^ (key & 7)) << 4)) = lo;
    *reinterpret_cast<uint4*>(at + (((piece + 1) ^ (key & 7)) << 4)) = hi;
  }
}

// Row `r` of a query tile in the same layout, bf16, to fp16 times 2^n, with the largest in [2^14, 2^15): exact but for elements
// below 2^-31 of it, off by 2^-39 of it at most. Returns 2^-n.
__device__ __forceinline__ float row_to_f16(unsigned char* tile, int rows, int r) {
  float top = 0.f;
#pragma unroll 4
  for (int i = 0; i < 16; ++i) {
    const uint4 w = *reinterpret_cast<const uint4*>(tile + (i >> 3) * (rows * 128) + r * 128 + (((i & 7) ^ (r & 7)) << 4));
    const uint32_t in[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const float a = fabsf(__uint_as_float(in[j] << 16)), b = fabsf(__uint_as_float(in[j] & 0xffff0000u));
      top = fmaxf(top, fmaxf(a < INFINITY ? a : 0.f, b < INFINITY ? b : 0.f));
    }
  }
  const int n = top == 0.f ? 0 : min(126, 14 + 127 - (int)(__float_as_uint(top) >> 23));
  const float up = __uint_as_float((uint32_t)(127 + n) << 23);
#pragma unroll 4
  for (int i = 0; i < 16; ++i) {
    uint4* at = reinterpret_cast<uint4*>(tile + (i >> 3) * (rows * 128) + r * 128 + (((i & 7) ^ (r & 7)) << 4));
    const uint4 w = *at;
    const uint32_t in[4] = {w.x, w.y, w.z, w.w};
    uint32_t y[4];
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const __half2 h = __floats2half2_rn(__uint_as_float(in[j] << 16) * up, __uint_as_float(in[j] & 0xffff0000u) * up);
      y[j] = reinterpret_cast<const uint32_t&>(h);
    }
    *at = make_uint4(y[0], y[1], y[2], y[3]);
  }
  return __uint_as_float((uint32_t)max(127 - n, 1) << 23);
}

// Instruction descriptor, kind::f16: fp16 A and B (K-major), fp32 accumulator, M x N.
__host__ __device__ constexpr uint32_t idesc_f16_f32(int M, int N) {
  return (1u << 4) | ((uint32_t)(N >> 3) << 17) | ((uint32_t)(M >> 4) << 24);
}

}  // namespace vr
