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
__device__ __forceinline__ float power_of_two(int e) { return __int_as_float((e + 127) << 23); }
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
// 16 codes as fp16, and the largest size of them (before their scale; NaN is none).
__device__ __forceinline__ void codes_f16(const uint4& c, __half2 (&h)[8]) {
    const uint32_t w[4] = {c.x, c.y, c.z, c.w};
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const uint32_t f = e4m3_to_f16x2(i & 1 ? w[i >> 1] >> 16 : w[i >> 1]);
        h[i] = *reinterpret_cast<const __half2*>(&f);
    }
}
__device__ __forceinline__ float code_size(const uint4& c) {
    __half2 h[8];
    codes_f16(c, h);
    __half2 m = __habs2(h[0]);
#pragma unroll
    for (int i = 1; i < 8; ++i) m = __hmax2(m, __habs2(h[i]));
    const float a = __low2float(m), b = __high2float(m);
    return fmaxf(fmaxf(a, b), 0.f);
}
// 16 codes of scale s as codes of the scale 2^e: their products with the ratio, which
// fp16 holds exactly for ratios down to 2^-15 (codes are multiples of 2^-9, fp16 numbers
// of 2^-24), rounded once.
__device__ __forceinline__ uint4 rescaled(const uint4& c, float s, int e) {
    const int k = (__float_as_int(s) >> 23) - 127 - e;
    if (k > 15 || k < -15) return make_uint4(to_e4m3(e4m3_values(c.x, s), e), to_e4m3(e4m3_values(c.y, s), e),
                                             to_e4m3(e4m3_values(c.z, s), e), to_e4m3(e4m3_values(c.w, s), e));
    const __half2 f = __float2half2_rn(power_of_two(k));
    __half2 h[8];
    codes_f16(c, h);
    uint32_t w[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const __half2 x = __hmul2(h[i], f);
        asm("{\n\t.reg .b16 t;\n\tcvt.rn.satfinite.e4m3x2.f16x2 t, %1;\n\tcvt.u32.u16 %0, t;\n\t}"
            : "=r"(w[i])
            : "r"(*reinterpret_cast<const uint32_t*>(&x)));
    }
    return make_uint4(w[0] | w[1] << 16, w[2] | w[3] << 16, w[4] | w[5] << 16, w[6] | w[7] << 16);
}
// Exponent of the scale for a largest size: size = m 2^k, 1 <= m < 2, against
// 448 = 1.75 * 2^8.
__device__ __forceinline__ int scale_exponent(float size) {
    const int bits = __float_as_int(size);
    const int e = (bits >> 23) - 127 - 8 + ((bits & 0x7fffff) > 0x600000 ? 1 : 0);
    return max(e, kLeastScale);
}
// Largest over the warp (sizes are not negative: their bits order as integers).
__device__ __forceinline__ float warp_size(float s) {
    return __uint_as_float(__reduce_max_sync(0xffffffffu, __float_as_uint(s)));
}

}  // namespace dev
}  // namespace sq
