// Paged attention on tcgen05: what the kernels share (internal).
#pragma once

#include "common.cuh"

namespace vr {

__device__ __forceinline__ bool elect_one() {
  uint32_t p;
  asm volatile("{\n .reg .pred p;\n elect.sync _|p, 0xffffffff;\n selp.u32 %0, 1, 0, p;\n}\n" : "=r"(p));
  return p != 0;
}
// D[tmem] (+)= A[tmem] * B[smem]^T (A: bf16 pairs, row = lane, 8 columns per K = 16), issued by one thread.
__device__ __forceinline__ void tc_mma_bf16_ts(uint32_t d_tmem, uint32_t a_tmem, uint64_t b, uint32_t idesc, uint32_t accumulate) {
  asm volatile(
      "{\n .reg .pred p;\n setp.ne.b32 p, %4, 0;\n"
      " tcgen05.mma.cta_group::1.kind::f16 [%0], [%1], %2, %3, p;\n}\n"
      ::"r"(d_tmem), "r"(a_tmem), "l"(b), "r"(idesc), "r"(accumulate) : "memory");
}
// 64 fp32 columns of this warp's 32 TMEM lanes.
__device__ __forceinline__ void tmem_ld64(uint32_t taddr, float (&v)[64]) {
  asm volatile(
      "tcgen05.ld.sync.aligned.32x32b.x64.b32 {"
      "%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,"
      "%16,%17,%18,%19,%20,%21,%22,%23,%24,%25,%26,%27,%28,%29,%30,%31,"
      "%32,%33,%34,%35,%36,%37,%38,%39,%40,%41,%42,%43,%44,%45,%46,%47,"
      "%48,%49,%50,%51,%52,%53,%54,%55,%56,%57,%58,%59,%60,%61,%62,%63"
      "}, [%64];\n tcgen05.wait::ld.sync.aligned;\n"
      : "=f"(v[0]), "=f"(v[1]), "=f"(v[2]), "=f"(v[3]), "=f"(v[4]), "=f"(v[5]), "=f"(v[6]), "=f"(v[7]),
        "=f"(v[8]), "=f"(v[9]), "=f"(v[10]), "=f"(v[11]), "=f"(v[12]), "=f"(v[13]), "=f"(v[14]), "=f"(v[15]),
        "=f"(v[16]), "=f"(v[17]), "=f"(v[18]), "=f"(v[19]), "=f"(v[20]), "=f"(v[21]), "=f"(v[22]), "=f"(v[23]),
        "=f"(v[24]), "=f"(v[25]), "=f"(v[26]), "=f"(v[27]), "=f"(v[28]), "=f"(v[29]), "=f"(v[30]), "=f"(v[31]),
        "=f"(v[32]), "=f"(v[33]), "=f"(v[34]), "=f"(v[35]), "=f"(v[36]), "=f"(v[37]), "=f"(v[38]), "=f"(v[39]),
        "=f"(v[40]), "=f"(v[41]), "=f"(v[42]), "=f"(v[43]), "=f"(v[44]), "=f"(v[45]), "=f"(v[46]), "=f"(v[47]),
        "=f"(v[48]), "=f"(v[49]), "=f"(v[50]), "=f"(v[51]), "=f"(v[52]), "=f"(v[53]), "=f"(v[54]), "=f"(v[55]),
        "=f"(v[56]), "=f"(v[57]), "=f"(v[58]), "=f"(v[59]), "=f"(v[60]), "=f"(v[61]), "=f"(v[62]), "=f"(v[63])
      : "r"(taddr) : "memory");
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
__device__ __forceinline__ void tma_load_3d(uint32_t dst, const void* tmap, int x, int y, int z, uint64_t* bar) {
  asm volatile(
      "cp.async.bulk.tensor.3d.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3, %4}], [%5];\n"
      ::"r"(dst), "l"(tmap), "r"(x), "r"(y), "r"(z), "r"(smem_addr(bar)) : "memory");
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

// Row `r` of a query tile in the same layout, bf16, to fp16 times 2^n, with the largest in [2^14, 2^15) (so exact down to 2^-38 of
// it); 2^-n.
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
