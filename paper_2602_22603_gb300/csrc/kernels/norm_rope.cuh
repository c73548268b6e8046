// A row of a head in a warp's registers: its norm, the rotation of its pairs, and
// the loads of what both take (see norm_rope.cu).
#pragma once

#include "operators.hpp"
#include "ptx.cuh"

namespace sq {
namespace dev {
namespace {

template <int D>
struct NormCfg {
    static constexpr int kLanes = D / 8;     // lanes of a row
    static constexpr int kGroups = 32 / kLanes;  // rows a warp holds at once
};

typedef uint64_t f32x2;  // two floats, the first in the low half
__device__ __forceinline__ f32x2 f2(float a, float b) {
    f32x2 r;
    asm("mov.b64 %0, {%1, %2};" : "=l"(r) : "f"(a), "f"(b));
    return r;
}
__device__ __forceinline__ float2 un2(f32x2 v) {
    float2 r;
    asm("mov.b64 {%0, %1}, %2;" : "=f"(r.x), "=f"(r.y) : "l"(v));
    return r;
}
__device__ __forceinline__ f32x2 fma2(f32x2 a, f32x2 b, f32x2 c) {
    f32x2 d;
    asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(d) : "l"(a), "l"(b), "l"(c));
    return d;
}
__device__ __forceinline__ f32x2 mul2(f32x2 a, f32x2 b) {
    f32x2 d;
    asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(d) : "l"(a), "l"(b));
    return d;
}
__device__ __forceinline__ f32x2 swap2(f32x2 v) {
    const float2 x = un2(v);
    return f2(x.y, x.x);
}
__device__ __forceinline__ f32x2 unpack2(uint32_t w) {
    return f2(__uint_as_float(w << 16), __uint_as_float(w & 0xffff0000u));
}
__device__ __forceinline__ uint32_t pack2(f32x2 v) {
    const float2 x = un2(v);
    return pack_bf16x2(x.x, x.y);
}

// Streaming loads (read once).
__device__ __forceinline__ uint2 ld_half_row(const __nv_bfloat16* p) {
    uint2 v;
    asm volatile("ld.global.nc.L1::no_allocate.v2.u32 {%0, %1}, [%2];" : "=r"(v.x), "=r"(v.y) : "l"(p));
    return v;
}
__device__ __forceinline__ uint4 ld_row(const __nv_bfloat16* p) {
    uint4 v;
    asm volatile("ld.global.nc.L1::no_allocate.v4.u32 {%0, %1, %2, %3}, [%4];"
                 : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w)
                 : "l"(p));
    return v;
}

// The eight elements a lane has of every row: f .. f + 3 and g .. g + 3.
struct Lane {
    int f, g;
    int pair;   // first of its four pairs in the table
    bool on;    // its elements turn
    template <bool kPairs>
    __device__ __forceinline__ void init(int l, int rot) {
        on = 8 * l < rot;  // (rot is a multiple of 16)
        pair = 4 * l;
        f = !kPairs && on ? 4 * l : 8 * l;
        g = !kPairs && on ? rot / 2 + 4 * l : 8 * l + 4;
    }
    // the part of a pair's other: none where the elements do not turn (a sine of 0
    // times an infinity is NaN)
    __device__ __forceinline__ f32x2 turned(f32x2 v) const { return on ? v : 0; }
};

// Eight values of a lane as pairs: f's, then g's.
struct Eight {
    f32x2 v[4];
    __device__ __forceinline__ void set(uint2 a, uint2 b) {
        v[0] = unpack2(a.x);
        v[1] = unpack2(a.y);
        v[2] = unpack2(b.x);
        v[3] = unpack2(b.y);
    }
    // what each element turns with
    template <bool kPairs>
    __device__ __forceinline__ f32x2 other(int i) const {
        return kPairs ? swap2(v[i]) : v[i ^ 2];
    }
};

// Four weights of an element type (ones where there are none).
__device__ __forceinline__ void load_weights4(const void* w, int f32, int e, f32x2& a, f32x2& b) {
    if (!w) {
        a = b = f2(1.f, 1.f);
    } else if (f32) {
        const float4 x = __ldg(reinterpret_cast<const float4*>(reinterpret_cast<const float*>(w) + e));
        a = f2(x.x, x.y);
        b = f2(x.z, x.w);
    } else {
        const uint2 x = __ldg(reinterpret_cast<const uint2*>(reinterpret_cast<const __nv_bfloat16*>(w) + e));
        a = unpack2(x.x);
        b = unpack2(x.y);
    }
}
__device__ __forceinline__ void load_weights(const void* w, int f32, const Lane& ln, Eight& x) {
    load_weights4(w, f32, ln.f, x.v[0], x.v[1]);
    load_weights4(w, f32, ln.g, x.v[2], x.v[3]);
}

// Cosines and sines of a lane's elements at one position (the sine negative where
// an element is its pair's first), 1 and 0 for those that do not turn.
struct Turn {
    f32x2 c[4], s[4];
};
// `pos` is inside the table.
template <bool kPairs>
__device__ __forceinline__ void load_turn(Turn& t, const float2* rope, int pos, int rot, const Lane& ln) {
    if (!ln.on) {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            t.c[i] = f2(1.f, 1.f);
            t.s[i] = f2(0.f, 0.f);
        }
        return;
    }
    const float4* p = reinterpret_cast<const float4*>(rope + (int64_t)pos * (rot >> 1) + ln.pair);
    const float4 a = __ldg(p), b = __ldg(p + 1);  // c0 s0 c1 s1, c2 s2 c3 s3
    if (kPairs) {
        t.c[0] = f2(a.x, a.x);
        t.c[1] = f2(a.z, a.z);
        t.c[2] = f2(b.x, b.x);
        t.c[3] = f2(b.z, b.z);
        t.s[0] = f2(-a.y, a.y);
        t.s[1] = f2(-a.w, a.w);
        t.s[2] = f2(-b.y, b.y);
        t.s[3] = f2(-b.w, b.w);
    } else {
        t.c[0] = t.c[2] = f2(a.x, a.z);
        t.c[1] = t.c[3] = f2(b.x, b.z);
        t.s[2] = f2(a.y, a.w);
        t.s[3] = f2(b.y, b.w);
        t.s[0] = f2(-a.y, -a.w);
        t.s[1] = f2(-b.y, -b.w);
    }
}

// Sum over the lanes of a row.
template <int D>
__device__ __forceinline__ float row_sum(f32x2 v) {
    const float2 p = un2(v);
    float x = p.x + p.y;
#pragma unroll
    for (int o = NormCfg<D>::kLanes / 2; o > 0; o >>= 1) x += __shfl_xor_sync(0xffffffffu, x, o);
    return x;
}

// A token's position for the table: one outside it is flagged and read as 0.
__device__ __forceinline__ int checked_pos(int pos, int max_pos, int* err) {
    if ((uint32_t)pos < (uint32_t)max_pos) return pos;
    set_error(err, kErrBounds);
    return 0;
}

}  // namespace
}  // namespace dev
}  // namespace sq
