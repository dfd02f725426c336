// Values of a cache of four bits.  A code's lowest three bits stand for 0, 0.5, 1, 1.5, 2, 3, 4, 6, the highest one for the sign; a group's
// scale byte s for 2^(s - 127), 255 for not a number.  A value is an amount times a power of two: bfloat16 holds it as it is.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "spec_internal.h"

namespace specdraft {

// eight codes of one group, the first in the lowest bits, as bfloat16: the conversion takes the exponent of its scale only, and gives
// every value of every scale byte as it is defined, subnormal ones among them
__device__ __forceinline__ u32x4 unpack_scaled(uint32_t codes, float scale) {
  u32x4 r;
  r[0] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, scale, 0));
  r[1] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, scale, 1));
  r[2] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, scale, 2));
  r[3] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, scale, 3));
  return r;
}
__device__ __forceinline__ u32x4 unpack_word(uint32_t codes, uint32_t scale_byte) { return unpack_scaled(codes, __uint_as_float(scale_byte << 23)); }

}  // namespace specdraft
