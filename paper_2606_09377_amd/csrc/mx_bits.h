// 4-bit values with a power of two for every 32 of them (vcrown.h, vcr_mx), in registers.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "split_bf16.h"

namespace vcr {

// the float of a scale byte, as the conversions take it
__device__ __forceinline__ float mx_scale(uint32_t byte) {
  return __builtin_bit_cast(float, byte == 255 ? 0x7fc00000u : byte == 0 ? 0x00400000u : byte << 23);
}
// eight values, exact
__device__ __forceinline__ uint4 mx_to_bf16(uint32_t u, float s) {
  auto c = [](auto v) { return __builtin_bit_cast(uint32_t, v); };
  return make_uint4(c(__builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(u, s, 0)), c(__builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(u, s, 1)),
                    c(__builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(u, s, 2)), c(__builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(u, s, 3)));
}

}  // namespace vcr
