// e4m3 codes with a power of two -> bf16, for the kernels that read an 8-bit cache.
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
#endif

}  // namespace amskv
