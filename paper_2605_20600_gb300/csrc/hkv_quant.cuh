// The 8- and 4-bit row format of include/hkv_serve.h on the device: groups of
// 32 channels, a bf16 scale each, biased codes.
#pragma once

#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <stdint.h>

#include "hkv_device.cuh"

namespace hkv {

template <int D, int BITS>
struct QRow {
  static constexpr int kBytes = D * BITS / 8;       // codes of a K or V row
  static constexpr int kGroups = D / 32;
  static constexpr int kScaleBytes = kGroups * 2;
  static constexpr int kBias = BITS == 8 ? 128 : 8;
  static constexpr int kMax = BITS == 8 ? 127 : 7;
};

// 8 neighbouring values of a plain row (16-byte aligned in bf16, 32-byte in fp32)
template <typename T>
__device__ __forceinline__ void load8(const void *p, float *x);
template <>
__device__ __forceinline__ void load8<float>(const void *p, float *x) {
  Elem<float>::unpack(reinterpret_cast<const uint4 *>(p)[0], x);
  Elem<float>::unpack(reinterpret_cast<const uint4 *>(p)[1], x + 4);
}
template <>
__device__ __forceinline__ void load8<__nv_bfloat16>(const void *p, float *x) {
  Elem<__nv_bfloat16>::unpack(*reinterpret_cast<const uint4 *>(p), x);
}

__device__ __forceinline__ float bf16_bits_to_float(uint32_t b) {
  return __uint_as_float(b << 16);
}

// Quantises a group of 32 values held by four neighbouring lanes (8 each, in
// channel order; the four call together, `mask` names the lanes of the warp
// that call). Returns the scale's bf16 bits (the same in the four lanes) and
// leaves this lane's biased codes in lo and hi: 8 bits, bytes of lo then hi;
// 4 bits, nibbles of lo. The magnitudes are compared as integers, so that a
// NaN or an infinity in the group shows (its bits are the largest).
template <int BITS>
__device__ __forceinline__ uint32_t quant_group(const float *x, uint32_t mask, uint32_t &lo,
                                                uint32_t &hi) {
  constexpr int kMax = BITS == 8 ? 127 : 7, kBias = BITS == 8 ? 128 : 8;
  uint32_t a = 0;
#pragma unroll
  for (int j = 0; j < 8; ++j) a = max(a, __float_as_uint(x[j]) & 0x7FFFFFFFu);
  a = max(a, __shfl_xor_sync(mask, a, 1));
  a = max(a, __shfl_xor_sync(mask, a, 2));
  const bool finite = a < 0x7F800000u;
  const float q = __fdiv_rn(__uint_as_float(a), (float)kMax);
  const uint32_t sb = finite ? (uint32_t)__bfloat16_as_ushort(__float2bfloat16_rn(q)) : 0x7FC0u;
  const float s = bf16_bits_to_float(sb);
  lo = hi = 0;
#pragma unroll
  for (int j = 0; j < 8; ++j) {
    int c = 0;
    if (s > 0.f) c = max(-kMax, min(kMax, __float2int_rn(__fdiv_rn(x[j], s))));
    const uint32_t b = (uint32_t)(c + kBias);
    if (BITS == 4) lo |= b << (4 * j);
    else if (j < 4) lo |= b << (8 * j);
    else hi |= b << (8 * (j - 4));
  }
  return sb;
}

}  // namespace hkv
