// Codes with a power of two -> bf16, for the kernels that read a cache of 8 bits (e4m3) or of 4 (e2m1).
#pragma once
#include "amskv_internal.hpp"

namespace amskv {

typedef unsigned int u32x2 __attribute__((ext_vector_type(2)));
typedef unsigned int u32x4 __attribute__((ext_vector_type(4)));

#if defined(__HIPCC__)
// 8 codes times scale (a power of two) as 8 bf16 numbers; exact: a code has 4 significant bits
__device__ __forceinline__ u32x4 values8(const u32x2& codes, float scale) {
  u32x4 out;
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    out[2 * i] = __builtin_bit_cast(unsigned, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(codes[i], scale, false));
    out[2 * i + 1] = __builtin_bit_cast(unsigned, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(codes[i], scale, true));
  }
  return out;
}

// 8 codes of 4 bits times scale as 8 bf16 numbers; exact: a code has 2 significant bits, and its product is a bf16 number
__device__ __forceinline__ u32x4 values4(unsigned codes, float scale) {
  return u32x4{__builtin_bit_cast(unsigned, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, scale, 0)),
               __builtin_bit_cast(unsigned, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, scale, 1)),
               __builtin_bit_cast(unsigned, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, scale, 2)),
               __builtin_bit_cast(unsigned, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, scale, 3))};
}

// Into 4 bits.  The 32 channels of a group of a row share the least power of two 2^e, -100 <= e <= 125, with max |x| <= 7 * 2^e; x is held
// as the e2m1 number next to x * 2^-e (v_cvt_scalef32_pk_fp4_f32: to nearest, ties to even, what is beyond 6 as 6, the nearest up to
// 7).  A power of two because the conversions and the matrix instructions take one; of the rules that choose one this has the least mean
// error on normal values (rms 0.1120 of their size; max |x| <= 6 * 2^e: 0.1156).  7 * 2^e = 1.75 * 2^(e + 2); e <= 125 since
// 6 * 2^126 is no bf16 number.
__device__ __forceinline__ int group_exponent(float m) {
  const int bits = __float_as_int(m);
  const int e = (bits >> 23) - 127 - 2 + ((bits & 0x7fffff) > 0x600000 ? 1 : 0);
  return min(max(e, -100), 125);
}
// the first of each two in the low half of a byte; scale: 2^e
__device__ __forceinline__ unsigned codes4(const float (&x)[8], float scale) {
  unsigned c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(0, x[0], x[1], scale, 0);
  c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(c, x[2], x[3], scale, 1);
  c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(c, x[4], x[5], scale, 2);
  return __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(c, x[6], x[7], scale, 3);
}
// 2^(byte - 127), byte 1 .. 254
__device__ __forceinline__ float power_of_byte(unsigned byte) { return __builtin_bit_cast(float, byte << 23); }
#endif

}  // namespace amskv
