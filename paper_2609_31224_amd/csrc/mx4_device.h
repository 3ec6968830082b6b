// Device helpers of rows held in 4 bits (gfx950).
#pragma once

#include "device_common.h"
#include "mx4.h"

namespace a2t {
namespace {

// 8 elements' codes times their block's scale as bf16: exact, and NaN for a scale byte of 255
// (s: the byte as an fp32 exponent)
__device__ __forceinline__ u32x4 mx4_to_bf16(uint32_t code, float s) {
    return u32x4{__builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(code, s, 0)),
                 __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(code, s, 1)),
                 __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(code, s, 2)),
                 __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(code, s, 3))};
}

}  // namespace
}  // namespace a2t
