// e4m3 codes with a power of two -> bf16, for the kernels that read an 8-bit cache.
#pragma once
#include "amskv_internal.hpp"

namespace amskv {

typedef unsigned int u32x2 __attribute__((ext_vector_type(2)));
typedef unsigned int u32x4 __attribute__((ext_vector_type(4)));

#if defined(__HIPCC__)
// 16 codes times scale (a power of two) as 16 bf16 numbers, two vectors of 8; exact: a code has 4 significant bits
__device__ __forceinline__ void values16(const u32x4& codes, float scale, u32x4 (&out)[2]) {
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    out[i >> 1][2 * (i & 1)] = __builtin_bit_cast(unsigned, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(codes[i], scale, false));
    out[i >> 1][2 * (i & 1) + 1] = __builtin_bit_cast(unsigned, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(codes[i], scale, true));
  }
}
#endif

}  // namespace amskv
