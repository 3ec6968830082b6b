// Device helpers of rows held in 4 bits (gfx950).
#pragma once

#include "device_common.h"
#include "mx4.h"

namespace a2t {
namespace {

typedef int i32x8 __attribute__((ext_vector_type(8)));
typedef short i16x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x6 __attribute__((ext_vector_type(6)));
typedef float f32x2 __attribute__((ext_vector_type(2)));
typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef float f32x32 __attribute__((ext_vector_type(32)));
typedef _Float16 f16x2 __attribute__((ext_vector_type(2)));

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
    const f32x2 a = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4((uint32_t)code, s, 0);
    const f32x2 b = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4((uint32_t)code, s, 1);
    return byte == kMxNaN ? f32x4{__uint_as_float(0x7fc00000u), __uint_as_float(0x7fc00000u), __uint_as_float(0x7fc00000u), __uint_as_float(0x7fc00000u)}
                          : f32x4{a[0], a[1], b[0], b[1]};
}
__device__ __forceinline__ bool mx4_odd(int byte) { return (uint32_t)(byte - kMxF16Low) > (uint32_t)(kMxF16High - kMxF16Low); }
// v_cvt_pk_f16_f32, round to nearest even
__device__ __forceinline__ uint32_t mx4_pack_f16x2(float a, float b) {
    return __builtin_bit_cast(uint32_t, __builtin_convertvector((f32x2{a, b}), f16x2));
}

// global memory (a pointer picked by branches would be loaded from as a flat address)
__device__ __forceinline__ u32x4 gload16(const uint8_t* p) {
    return *reinterpret_cast<const __attribute__((address_space(1))) u32x4*>(reinterpret_cast<uintptr_t>(p));
}
__device__ __forceinline__ uint32_t gload4(const uint8_t* p) {
    return *reinterpret_cast<const __attribute__((address_space(1))) uint32_t*>(reinterpret_cast<uintptr_t>(p));
}
__device__ __forceinline__ int gload1(const uint8_t* p) {
    return *reinterpret_cast<const __attribute__((address_space(1))) uint8_t*>(reinterpret_cast<uintptr_t>(p));
}

// Rotates 8 dims of the lower half of a query row and their partners of the upper one, times s, to `lo` and `hi`.
__device__ __forceinline__ void mx4_rotate(const u32x4& a, const u32x4& a2, const float4 (&cs)[4], float s, float* lo, float* hi) {
    f32x4 yl[2], yh[2];
#pragma unroll
    for (int e = 0; e < 4; ++e) {
        const float lo0 = __uint_as_float(a[e] << 16), lo1 = __uint_as_float(a[e] & 0xffff0000u);
        const float hi0 = __uint_as_float(a2[e] << 16), hi1 = __uint_as_float(a2[e] & 0xffff0000u);
        yl[e / 2][2 * (e & 1)] = (lo0 * cs[e].x - hi0 * cs[e].y) * s;
        yl[e / 2][2 * (e & 1) + 1] = (lo1 * cs[e].z - hi1 * cs[e].w) * s;
        yh[e / 2][2 * (e & 1)] = (hi0 * cs[e].x + lo0 * cs[e].y) * s;
        yh[e / 2][2 * (e & 1) + 1] = (hi1 * cs[e].z + lo1 * cs[e].w) * s;
    }
#pragma unroll
    for (int e = 0; e < 2; ++e) {
        reinterpret_cast<f32x4*>(lo)[e] = yl[e];
        reinterpret_cast<f32x4*>(hi)[e] = yh[e];
    }
}
// A block of a rotated query, in LDS, as three e2m3 numbers an element: the largest magnitude becomes 3.875 to 7.75
// units (of e2m3's 7.5) of 2^(scale - 127), the scale byte that is returned; x[0] is off by up to 1/4
// unit, x[1], in units of 2^-kMxQueryStep[1], holds the rest to 1/128, and x[2] that one to 1/4096.
constexpr int kMxQueryParts = 3;
constexpr int kMxQueryStep[kMxQueryParts] = {0, 4, 9};
constexpr int kMxQueryLeast = 14;   // least scale byte (none goes below 0 where steps are taken off twice)
__device__ __forceinline__ int mx4_query(const float* block, u32x6 (&x)[kMxQueryParts]) {
    const f32x4* row = reinterpret_cast<const f32x4*>(block);
    f32x16 even, odd;   // the conversion interleaves its two operands
    uint32_t big = 0;
#pragma unroll
    for (int k = 0; k < 8; ++k) {
        const f32x4 y = row[k];
#pragma unroll
        for (int e = 0; e < 2; ++e) {
            even[2 * k + e] = y[2 * e];
            odd[2 * k + e] = y[2 * e + 1];
            big = max(big, max(__float_as_uint(y[2 * e]) & 0x7fffffffu, __float_as_uint(y[2 * e + 1]) & 0x7fffffffu));
        }
    }
#pragma unroll
    for (int p = 0; p < kMxQueryParts; ++p) x[p] = u32x6{0u, 0u, 0u, 0u, 0u, 0u};
    if (big >= 0x7f800000u) return kMxNaN;
    const int scale = max((int)((big + 0x80000u) >> 23) - 2, kMxQueryLeast);
    // (The conversions take several passes, and a result may not lie in their operands' registers, which the
    // compiler does not know: operands are kept until after them.)
#pragma unroll
    for (int p = 0; p < kMxQueryParts; ++p) {
        float unit = __uint_as_float((uint32_t)(scale - kMxQueryStep[p]) << 23);
        x[p] = __builtin_amdgcn_cvt_scalef32_2xpk16_fp6_f32(even, odd, unit);
        if (p + 1 < kMxQueryParts) {
            const f32x32 back = __builtin_amdgcn_cvt_scalef32_pk32_f32_fp6(x[p], unit);
#pragma unroll
            for (int e = 0; e < 16; ++e) {
                even[e] -= back[2 * e];
                odd[e] -= back[2 * e + 1];
            }
        }
        asm volatile("" : "+v"(unit), "+v"(x[p]), "+v"(even), "+v"(odd));
    }
    return scale;
}
// The scale of part p of a block with scale byte `scale`.
__device__ __forceinline__ int mx4_query_scale(int scale, int p) { return scale == kMxNaN ? scale : scale - kMxQueryStep[p]; }
__device__ __forceinline__ i32x8 mx4_operand(const u32x6& x) {
    return i32x8{(int)x[0], (int)x[1], (int)x[2], (int)x[3], (int)x[4], (int)x[5], 0, 0};
}

}  // namespace
}  // namespace a2t
