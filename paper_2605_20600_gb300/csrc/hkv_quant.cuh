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

// 2^15 + uu for the stored code uu: byte b of w (8 bits) or nibble n (4 bits).
// 0x4700uu00 is that fp32 number. Less 2^15 + bias it is the code c, exactly.
template <int BITS>
__device__ __forceinline__ float lifted(uint32_t w, int j) {
  if (BITS == 8) return __uint_as_float(__byte_perm(w, 0x47000000u, 0x7504 + (j << 4)));
  const uint32_t u = j < 2 ? w << (8 - 4 * j) : w >> (4 * j - 8);
  return __uint_as_float((u & 0xF00u) | 0x47000000u);
}
template <int BITS>
constexpr float kLift = 32768.f + (BITS == 8 ? 128.f : 8.f);

// Quantises a group of 32 values held by four neighbouring lanes (8 each, in
// channel order; the four call together, `mask` names them). Returns the
// scale's bf16 bits (the same in the four lanes) and leaves this lane's biased
// codes in lo and hi: 8 bits, bytes of lo then hi; 4 bits, nibbles of lo. The
// magnitudes are compared as integers, so that a NaN or an infinity in the
// group shows (its bits are the largest).
//
// bf16 values, without a division: x rcp(s) is within 2^-16 of x / s (at most
// 2^7 in magnitude), and one fma rounds it to a grid of 2^-12. A tie k + 1/2
// lies on the grid and is met exactly; any other quotient is more than 2^-10
// from a tie (x and s have 8 bits, so 2 x - (2 k + 1) s is at least a unit of
// 2 x or of s, which is 1/255 of it or more) and stays on its side; so rounding
// that to an integer, the sum with 1.5 * 2^23, rounds as x / s itself would be.
// a / M is at least 2^-16 (relative) from the midpoint of two bf16 numbers, so a
// product with 1 / M rounds alike. fp32 values, and groups whose scale is tiny,
// take the quotients.
template <typename T, int BITS>
__device__ __forceinline__ uint32_t quant_group(const float *x, uint32_t mask, uint32_t &lo,
                                                uint32_t &hi) {
  constexpr int kMax = BITS == 8 ? 127 : 7, kBias = BITS == 8 ? 128 : 8;
  uint32_t a = 0;
#pragma unroll
  for (int j = 0; j < 8; ++j) a = max(a, __float_as_uint(x[j]) & 0x7FFFFFFFu);
  a = max(a, __shfl_xor_sync(mask, a, 1));
  a = max(a, __shfl_xor_sync(mask, a, 2));
  uint32_t c[8];  // biased codes in the low bits, something above them
  float s;
  uint32_t sb;
  if (sizeof(T) == 2 && a >= 0x0E000000u && a < 0x7F800000u) {  // 2^-99 <= a, finite
    constexpr float kGrid = 2560.f, kInt = 12582912.f + kBias - kGrid;
    sb = __bfloat16_as_ushort(__float2bfloat16_rn(__uint_as_float(a) * (1.f / kMax)));
    s = bf16_bits_to_float(sb);
    float inv;
    asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(inv) : "f"(s));
#pragma unroll
    for (int j = 0; j < 8; ++j)
      c[j] = __float_as_uint(__fadd_rn(__fmaf_rn(x[j], inv, kGrid), kInt));
  } else {
    const bool finite = a < 0x7F800000u;
    const float q = __fdiv_rn(__uint_as_float(a), (float)kMax);
    sb = finite ? (uint32_t)__bfloat16_as_ushort(__float2bfloat16_rn(q)) : 0x7FC0u;
    s = bf16_bits_to_float(sb);
#pragma unroll
    for (int j = 0; j < 8; ++j)
      c[j] = (uint32_t)(kBias + (s > 0.f ? max(-kMax, min(kMax, __float2int_rn(__fdiv_rn(x[j], s))))
                                         : 0));
  }
  if (BITS == 8) {
    lo = __byte_perm(__byte_perm(c[0], c[1], 0x0040), __byte_perm(c[2], c[3], 0x0040), 0x5410);
    hi = __byte_perm(__byte_perm(c[4], c[5], 0x0040), __byte_perm(c[6], c[7], 0x0040), 0x5410);
  } else {
    lo = c[0] & 15u;
#pragma unroll
    for (int j = 1; j < 8; ++j) lo |= (c[j] & 15u) << (4 * j);
    hi = 0;
  }
  return sb;
}

// A running maximum before its first key: finite, so that keys whose scores are
// -inf (or that do not count) weigh nothing against it.
constexpr float kNoKey = -0x1.fffffep127f;

// Byte offset of the 16-byte piece `c` of row `r` in a tile: rows lie back to
// back, the pieces permuted so that the reads below spread over all banks.
template <int RB>
__device__ __forceinline__ int piece_at(int r, int c) {
  if (RB == 128) return r * 128 + ((c ^ (r & 7)) << 4);
  if (RB == 64) return r * 64 + ((c ^ ((r >> 1) & 3)) << 4);
  return r * 32 + ((c ^ ((r >> 2) & 1)) << 4);
}

// E neighbouring fp32 numbers of a partial result, past L1
template <int E>
__device__ __forceinline__ void load_row(const float *from, float (&o)[E]) {
  if (E == 4) {
    const float4 u = __ldcg(reinterpret_cast<const float4 *>(from));
    o[0] = u.x, o[1 % E] = u.y, o[2 % E] = u.z, o[3 % E] = u.w;
  } else {
    const float2 u = __ldcg(reinterpret_cast<const float2 *>(from));
    o[0] = u.x, o[1 % E] = u.y;
  }
}

}  // namespace hkv
