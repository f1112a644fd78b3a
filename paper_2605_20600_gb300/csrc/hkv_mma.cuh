// mma.sync m16n8k16 on bf16 tiles in shared memory, and the parts that fp32
// numbers enter it in.
#pragma once

#include <cuda_bf16.h>
#include <stdint.h>

#include "hkv_device.cuh"

namespace hkv {

// byte offset of 16-byte piece c of row r: pieces permuted over the banks
template <int D>
__device__ __forceinline__ int at16(int r, int c) {
  return r * (D * 2) + ((c ^ (r & 7)) << 4);
}

__device__ __forceinline__ void ldm4(uint32_t (&r)[4], uint32_t a) {
  asm volatile("ldmatrix.sync.aligned.m8n8.x4.shared.b16 {%0,%1,%2,%3}, [%4];"
               : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3])
               : "r"(a)
               : "memory");
}
__device__ __forceinline__ void ldm4t(uint32_t (&r)[4], uint32_t a) {
  asm volatile("ldmatrix.sync.aligned.m8n8.x4.trans.shared.b16 {%0,%1,%2,%3}, [%4];"
               : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3])
               : "r"(a)
               : "memory");
}
__device__ __forceinline__ void mma_bf16(float (&c)[4], const uint32_t (&a)[4], uint32_t b0,
                                         uint32_t b1) {
  asm volatile(
      "mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, "
      "{%8,%9}, {%0,%1,%2,%3};"
      : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
      : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}
// 16 bytes to shared memory, zeros where `on` is false (nothing is read then)
__device__ __forceinline__ void cp_async16_zfill(void *dst, const void *src, bool on) {
  asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(smem_u32(dst)), "l"(src),
               "r"(on ? 16 : 0)
               : "memory");
}
__device__ __forceinline__ uint32_t pack2(float lo, float hi) {
  const __nv_bfloat162 h = __floats2bfloat162_rn(lo, hi);
  return *reinterpret_cast<const uint32_t *>(&h);
}
// a pair of fp32 as bf16 parts of falling size; the remainder is exact. ANY: the
// first part stays finite where an element lies above the largest bf16 number
// (an infinity's parts hold a NaN, as a NaN's do).
template <bool ANY>
__device__ __forceinline__ void split2(float x, float y, uint32_t (&p)[3]) {
  constexpr float kMost = 0x1.fep127f;
#pragma unroll
  for (int j = 0; j < 3; ++j) {
    p[j] = ANY && j == 0 ? pack2(fminf(fmaxf(x, -kMost), kMost), fminf(fmaxf(y, -kMost), kMost))
                         : pack2(x, y);
    x -= __uint_as_float(p[j] << 16);
    y -= __uint_as_float(p[j] & 0xFFFF0000u);
  }
}

}  // namespace hkv
