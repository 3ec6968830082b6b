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

// The same as fp16, for scale bytes from kMxF16Low to kMxF16High: exact too (fp16 holds multiples of
// 2^-24 up to 65504; elements are multiples of half a scale up to six of them).
constexpr int kMxF16Low = 127 - 23, kMxF16High = 127 + 13;
__device__ __forceinline__ u32x4 mx4_to_f16(uint32_t code, float s) {
    return u32x4{__builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp4(code, s, 0)),
                 __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp4(code, s, 1)),
                 __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp4(code, s, 2)),
                 __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp4(code, s, 3))};
}
// 4 elements as fp32, for any scale byte
__device__ __forceinline__ f32x4 mx4_to_f32(int code, int byte) {
    const float s = __uint_as_float((uint32_t)byte << 23);
    typedef float f32x2 __attribute__((ext_vector_type(2)));
    const f32x2 a = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4((uint32_t)code, s, 0);
    const f32x2 b = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4((uint32_t)code, s, 1);
    return byte == kMxNaN ? f32x4{__uint_as_float(0x7fc00000u), __uint_as_float(0x7fc00000u), __uint_as_float(0x7fc00000u), __uint_as_float(0x7fc00000u)}
                          : f32x4{a[0], a[1], b[0], b[1]};
}
// v_cvt_pk_f16_f32, round to nearest even
__device__ __forceinline__ uint32_t mx4_pack_f16x2(float a, float b) {
    typedef float f32x2 __attribute__((ext_vector_type(2)));
    typedef _Float16 f16x2 __attribute__((ext_vector_type(2)));
    return __builtin_bit_cast(uint32_t, __builtin_convertvector((f32x2{a, b}), f16x2));
}

}  // namespace
}  // namespace a2t
