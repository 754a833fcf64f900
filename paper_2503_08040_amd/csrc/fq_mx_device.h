// What the kernels of microscaled 4-bit matrices share: sizes of the stored pieces, a group's scale, conversion.
#pragma once
#include "fq_device.h"

namespace fq {
namespace {

constexpr int kOperand = 1024;    // bytes of codes of 16 rows x 128
constexpr int kScaleBlock = 256;  // bytes of scales of 64 rows x 128

typedef uint32_t v4u __attribute__((ext_vector_type(4)));
// the same in memory at any element's address: global memory takes vector accesses of any alignment
typedef uint32_t v4u_at2 __attribute__((ext_vector_type(4), aligned(2)));
typedef uint32_t v2u_at2 __attribute__((ext_vector_type(2), aligned(2)));
typedef float v4f_at4 __attribute__((ext_vector_type(4), aligned(4)));
typedef uint16_t v2h __attribute__((ext_vector_type(2)));
typedef __bf16 v2bf __attribute__((ext_vector_type(2)));
typedef uint32_t v2u __attribute__((ext_vector_type(2)));

__device__ __forceinline__ uint32_t pk_max(uint32_t a, uint32_t b) {
  return __builtin_bit_cast(uint32_t, __builtin_elementwise_max(__builtin_bit_cast(v2h, a), __builtin_bit_cast(v2h, b)));
}

// maximum over the 4 lanes of a quad
__device__ __forceinline__ uint32_t quad_max(uint32_t v) {
  v = pk_max(v, (uint32_t)__builtin_amdgcn_mov_dpp((int)v, 0xB1, 0xF, 0xF, true));   // lanes 1, 0, 3, 2
  return pk_max(v, (uint32_t)__builtin_amdgcn_mov_dpp((int)v, 0x4E, 0xF, 0xF, true));   // lanes 2, 3, 0, 1
}

// maximum over the 4 lanes 16 apart
__device__ __forceinline__ uint32_t row_max(uint32_t v) {
  v2u s = __builtin_amdgcn_permlane32_swap(v, v, false, false);
  v = pk_max(s[0], s[1]);
  s = __builtin_amdgcn_permlane16_swap(v, v, false, false);
  return pk_max(s[0], s[1]);
}

// Scale byte of a group with largest magnitude m (bf16 bits without the sign).  bias 63 takes the next exponent if
// the mantissa is above 1.5; the smallest byte is 0.
__device__ __forceinline__ uint32_t scale_byte(uint32_t m, int bias) {
  const uint32_t e = (m + (uint32_t)bias) >> 7;
  return m >= 0x7F80u ? 255u : (e > 2u ? e : 2u) - 2u;
}

// 2^(byte - 127) as the conversions take it; 2^-127 is a subnormal number.
__device__ __forceinline__ float scale_value(uint32_t byte) { return __uint_as_float(byte ? byte << 23 : 0x00400000u); }

__device__ __forceinline__ uint32_t cvt_fp4(uint32_t old, uint32_t pair, float scale, int sel) {
  const v2bf v = __builtin_bit_cast(v2bf, pair);
  switch (sel) {
    case 0: return __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(old, v, scale, 0);
    case 1: return __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(old, v, scale, 1);
    case 2: return __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(old, v, scale, 2);
    default: return __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(old, v, scale, 3);
  }
}

}  // namespace
}  // namespace fq
