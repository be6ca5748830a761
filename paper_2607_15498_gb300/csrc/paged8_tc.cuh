// Paged attention on tcgen05: what the kernels share (internal).
#pragma once

#include "common.cuh"

namespace vr {

__device__ __forceinline__ bool elect_one() {
  uint32_t p;
  asm volatile("{\n .reg .pred p;\n elect.sync _|p, 0xffffffff;\n selp.u32 %0, 1, 0, p;\n}\n" : "=r"(p));
  return p != 0;
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

// Key `key` of a tile: its 128 codes as 128 bf16 times the scale 2^(byte - 127), zeros where it is not `there`. The tile is two panels
// of `rows` rows of 64 elements, 128-byte swizzle; the codes stand, swizzled as well, where the second half of the key's row will
// be, so a thread per key touches nothing of another's.
__device__ __forceinline__ void expand_row(unsigned char* tile, int rows, int key, bool there, uint32_t byte) {
  unsigned char* row = tile + key * 128;
  const uint32_t scale2 = byte * 0x00800080u;
  uint4 w[8];
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    w[i] = *reinterpret_cast<const uint4*>(row + rows * 128 + ((i ^ (key & 7)) << 4));
    if (!there) w[i] = make_uint4(0, 0, 0, 0);
  }
#pragma unroll
  for (int i = 0; i < 8; ++i) {                             // elements 16 i .. 16 i + 15
    uint4 lo, hi;
    expand16(w[i], scale2, lo, hi);
    unsigned char* at = row + (i >> 2) * (rows * 128);
    const int piece = 2 * (i & 3);
    *reinterpret_cast<uint4*>(at + ((piece ^ (key & 7)) << 4)) = lo;
    *reinterpret_cast<uint4*>(at + (((piece + 1) ^ (key & 7)) << 4)) = hi;
  }
}

}  // namespace vr
