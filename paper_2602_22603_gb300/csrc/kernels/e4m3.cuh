// e4m3 codes and the power-of-two scales of their blocks (see kv8.hpp).
#pragma once

#include <cuda_fp16.h>

#include "kv8.hpp"
#include "ptx.cuh"

namespace sq {
namespace dev {

// One thread of a converged warp.
__device__ __forceinline__ bool elect_one() {
    uint32_t on;
    asm volatile("{\n\t.reg .pred p;\n\telect.sync _|p, 0xffffffff;\n\tselp.u32 %0, 1, 0, p;\n\t}" : "=r"(on));
    return on != 0;
}

// Two codes (the low 16 bits) as fp16, exact: the first in the low half.
__device__ __forceinline__ uint32_t e4m3_to_f16x2(uint32_t two) {
    uint32_t r;
    asm("{\n\t.reg .b16 lo;\n\tcvt.u16.u32 lo, %1;\n\tcvt.rn.f16x2.e4m3x2 %0, lo;\n\t}" : "=r"(r) : "r"(two));
    return r;
}
__device__ __forceinline__ float2 f16x2_to_f32(uint32_t v) {
    return __half22float2(*reinterpret_cast<const __half2*>(&v));
}
// Four codes as values.
__device__ __forceinline__ float4 e4m3_values(uint32_t four, float scale) {
    const float2 a = f16x2_to_f32(e4m3_to_f16x2(four)), b = f16x2_to_f32(e4m3_to_f16x2(four >> 16));
    return make_float4(a.x * scale, a.y * scale, b.x * scale, b.y * scale);
}
// A value (already divided by its scale) for the conversion: what is not finite is
// NaN, and of the largest scale, 2^kMostScale, codes past 240 would stand for
// infinities.
__device__ __forceinline__ float e4m3_input(float x, float most) {
    return fabsf(x) <= 3.4028234e38f ? fminf(fmaxf(x, -most), most) : NAN;
}
// Two values of at most 448 or NaN as codes, to nearest even: a's in the low byte.
__device__ __forceinline__ uint32_t to_e4m3x2(float a, float b) {
    uint32_t r;
    asm("{\n\t.reg .b16 t;\n\tcvt.rn.satfinite.e4m3x2.f32 t, %2, %1;\n\tcvt.u32.u16 %0, t;\n\t}"
        : "=r"(r)
        : "f"(a), "f"(b));
    return r;
}
// Any two.
__device__ __forceinline__ uint32_t to_e4m3x2(float a, float b, float most) {
    return to_e4m3x2(e4m3_input(a, most), e4m3_input(b, most));
}
__device__ __forceinline__ uint32_t to_e4m3(const float4& v, int e) {
    const float inv = __int_as_float((127 - e) << 23), most = e < kMostScale ? 448.f : 240.f;
    return to_e4m3x2(v.x * inv, v.y * inv, most) | to_e4m3x2(v.z * inv, v.w * inv, most) << 16;
}

// The size of an element for its block's scale: of one that is not finite none.
__device__ __forceinline__ float finite_size(float x) {
    const float a = fabsf(x);
    return a <= 3.4028234e38f ? a : 0.f;
}
__device__ __forceinline__ float finite_size(const float4& v) {
    return fmaxf(fmaxf(finite_size(v.x), finite_size(v.y)), fmaxf(finite_size(v.z), finite_size(v.w)));
}
// Exponent of the scale for a largest size: size = m 2^k, 1 <= m < 2, against
// 448 = 1.75 * 2^8.
__device__ __forceinline__ int scale_exponent(float size) {
    const int bits = __float_as_int(size);
    const int e = (bits >> 23) - 127 - 8 + ((bits & 0x7fffff) > 0x600000 ? 1 : 0);
    return max(e, kLeastScale);
}
__device__ __forceinline__ float power_of_two(int e) { return __int_as_float((e + 127) << 23); }
// Largest over the warp (sizes are not negative: their bits order as integers).
__device__ __forceinline__ float warp_size(float s) {
    return __uint_as_float(__reduce_max_sync(0xffffffffu, __float_as_uint(s)));
}

}  // namespace dev
}  // namespace sq
