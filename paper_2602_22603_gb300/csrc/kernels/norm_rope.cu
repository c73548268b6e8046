// Norms of queries and keys for each head with the position rotation in the
// same pass, forwards (to tensors, or keys and values straight into the paged
// pool) and backwards.
//
// Forwards, for every token and head with a row x of D elements:
//     r = (mean(x^2) + eps)^(-1/2),   y = w * (x r),
// then the first `rot` dimensions of y turn by the token's position, pairs
// (a, b) -> (a c - b s, b c + a s) with (c, s) from the caller's table; a pair is
// (e, e + rot / 2), or neighbours (2e, 2e + 1).  Everything is fp32 and rounded
// once, to the bf16 that the attention kernels read.
//
// Backwards, from dz of the rotated row: dy = dz turned back (the transpose of a
// rotation), dn = w dy, dx = r (dn - x r * mean(dn * x r)), dw = sum over tokens
// and heads of dy * x r.
//
// What bounds it: HBM.  Every row is read once and written once, 2 D bytes each
// way, and the arithmetic per row (~10 fp32 operations an element) is a third of
// what the SMs do meanwhile.  A row takes D / 8 lanes with a 16-byte vector each,
// so its sum of squares is 3 or 4 shuffles and a half-pair's partner one shuffle
// an element; a warp has one token's table rows in registers and kUnroll rows of
// each lane group in flight.
#include <algorithm>
#include <type_traits>

#include "operators.hpp"
#include "ptx.cuh"

namespace sq {
namespace {

using namespace dev;

constexpr int kNormThreads = 256;
constexpr int kUnroll = 4;  // rows of a lane group in flight

template <int D>
struct NormCfg {
    static constexpr int kLanes = D / 8;                 // lanes of a row
    static constexpr int kGroups = 32 / kLanes;          // rows a warp holds at once
    static constexpr int kTaskRows = kGroups * kUnroll;  // rows of a warp's task
};

__device__ __forceinline__ void unpack8(const uint4& v, float (&x)[8]) {
    const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        x[2 * i] = __uint_as_float(w[i] << 16);
        x[2 * i + 1] = __uint_as_float(w[i] & 0xffff0000u);
    }
}

__device__ __forceinline__ uint4 pack8(const float (&x)[8]) {
    return make_uint4(pack_bf16x2(x[0], x[1]), pack_bf16x2(x[2], x[3]), pack_bf16x2(x[4], x[5]),
                      pack_bf16x2(x[6], x[7]));
}

// Streaming 16-byte load (read once).
__device__ __forceinline__ uint4 ld_row(const void* p) {
    uint4 v;
    asm volatile("ld.global.nc.L1::no_allocate.v4.u32 {%0, %1, %2, %3}, [%4];"
                 : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w)
                 : "l"(p));
    return v;
}

// The norm's weights of elements e0 .. e0 + 7 (ones where there are none).
__device__ __forceinline__ void load_weights(const void* w, int f32, int e0, float (&x)[8]) {
    if (!w) {
#pragma unroll
        for (int i = 0; i < 8; ++i) x[i] = 1.f;
    } else if (f32) {
        const float4* p = reinterpret_cast<const float4*>(reinterpret_cast<const float*>(w) + e0);
        const float4 a = __ldg(p), b = __ldg(p + 1);
        x[0] = a.x; x[1] = a.y; x[2] = a.z; x[3] = a.w;
        x[4] = b.x; x[5] = b.y; x[6] = b.z; x[7] = b.w;
    } else {
        unpack8(__ldg(reinterpret_cast<const uint4*>(reinterpret_cast<const __nv_bfloat16*>(w) + e0)), x);
    }
}

// A lane's part of the rotation at one position: the cosine and sine of each of
// its elements (of pairs of neighbours: of elements 2 i and 2 i + 1), the sine
// negative where the element is its pair's first, and the lane holding the other
// halves.
struct Turn {
    float c[8], s[8];
    int partner;
    bool on;  // this lane's elements turn
};

// `pos` is inside the table.  `group0`: the row's first lane.
__device__ __forceinline__ void load_turn(Turn& t, const float2* rope, int pos, int rot, int interleaved,
                                          int e0, int group0) {
    t.on = e0 < rot;
    t.partner = group0 + e0 / 8;
    if (!t.on) return;
    const int half = rot >> 1;  // a multiple of 8
    const float2* row = rope + (int64_t)pos * half;
    if (interleaved) {
        const float4* p = reinterpret_cast<const float4*>(row + e0 / 2);
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            const float4 v = __ldg(p + i);
            t.c[4 * i] = t.c[4 * i + 1] = v.x;
            t.s[4 * i] = -v.y;
            t.s[4 * i + 1] = v.y;
            t.c[4 * i + 2] = t.c[4 * i + 3] = v.z;
            t.s[4 * i + 2] = -v.w;
            t.s[4 * i + 3] = v.w;
        }
        return;
    }
    const bool first = e0 < half;
    t.partner = group0 + (first ? e0 + half : e0 - half) / 8;
    const float4* p = reinterpret_cast<const float4*>(row + (first ? e0 : e0 - half));
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const float4 v = __ldg(p + i);
        t.c[2 * i] = v.x;
        t.s[2 * i] = first ? -v.y : v.y;
        t.c[2 * i + 1] = v.z;
        t.s[2 * i + 1] = first ? -v.w : v.w;
    }
}

// y turned by the position (kBack: turned back, the transpose).  Every lane of
// the warp calls it.
template <bool kBack>
__device__ __forceinline__ void turn(const Turn& t, int interleaved, float (&y)[8]) {
    float o[8];
    if (interleaved) {
#pragma unroll
        for (int i = 0; i < 8; ++i) o[i] = y[i ^ 1];
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i) o[i] = __shfl_sync(0xffffffffu, y[i], t.partner);
    }
    if (t.on) {
#pragma unroll
        for (int i = 0; i < 8; ++i) y[i] = kBack ? y[i] * t.c[i] - o[i] * t.s[i] : y[i] * t.c[i] + o[i] * t.s[i];
    }
}

// Sum over the lanes of a row.
template <int D>
__device__ __forceinline__ float row_sum(float x) {
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

// One warp: kTaskRows of a token's rows (its query heads, its key heads, and
// with kStore its value heads, which are copied).
template <int D, bool kStore, typename Args>
__global__ void __launch_bounds__(kNormThreads)
    sq_norm_rope_kernel(const __grid_constant__ Args a) {
    using C = NormCfg<D>;
    constexpr bool kInline = std::is_same<Args, NormRopeInlineArgs>::value;
    grid_dependency_wait();
    grid_launch_dependents();
    const int lane = threadIdx.x & 31;
    const int n_rows = a.Hq + (kStore ? 2 : 1) * a.Hkv;
    const unsigned chunks = (unsigned)(n_rows + C::kTaskRows - 1) / C::kTaskRows;
    // (n x chunks fits: the rows of as many tokens would not fit the device)
    const unsigned task = blockIdx.x * (kNormThreads / 32) + (threadIdx.x >> 5);
    const unsigned t = task / chunks;
    if (t >= (unsigned)a.n) return;
    const int sub = lane / C::kLanes, e0 = (lane % C::kLanes) * 8;
    const int row0 = (int)(task - t * chunks) * C::kTaskRows + sub;
    uint4 raw[kUnroll];
#pragma unroll
    for (int u = 0; u < kUnroll; ++u) {
        const int h = row0 + u * C::kGroups;
        const __nv_bfloat16* p = h < a.Hq ? a.q + t * a.q_stride + (int64_t)h * D
                                 : h < a.Hq + a.Hkv
                                     ? a.k + t * a.k_stride + (int64_t)(h - a.Hq) * D
                                     : a.v + t * a.v_stride + (int64_t)(h - a.Hq - a.Hkv) * D;
        raw[u] = h < n_rows ? ld_row(p + e0) : make_uint4(0, 0, 0, 0);
    }
    RowPlace place = {0, 0};
    if constexpr (kStore) {
        if constexpr (kInline) place = a.inline_place[t];
        else place = a.places[t];
    }
    Turn tn;
    {
        int pos = a.positions ? __ldg(&a.positions[t]) : place.pos;
        if (a.rot > 0) pos = checked_pos(pos, a.max_pos, a.err);
        load_turn(tn, a.rope, pos, a.rot, a.interleaved, e0, sub * C::kLanes);
    }
    float wq[8], wk[8];
    load_weights(a.q_weight, a.weight_f32, e0, wq);
    load_weights(a.k_weight, a.weight_f32, e0, wk);
    __nv_bfloat16* kv_row = nullptr;  // the token's row of head 0 of K in the pool
    if constexpr (kStore) {
        const int lp = __ffs(a.P) - 1;
        const int64_t page = place.row >> lp;
        if (place.row >= 0 && page < a.num_pages)
            kv_row = a.pool + (((int64_t)a.layer * a.num_pages + page) * 2 * a.Hkv * a.P +
                               (place.row & (a.P - 1))) * D;
        else set_error(a.err, kErrBounds);
    }
#pragma unroll
    for (int u = 0; u < kUnroll; ++u) {
        const int h = row0 + u * C::kGroups;
        if (row0 - sub + u * C::kGroups >= n_rows) break;  // (warp-uniform)
        const bool is_k = h >= a.Hq, is_v = kStore && h >= a.Hq + a.Hkv;
        float y[8];
        unpack8(raw[u], y);
        float ss = 0.f;
#pragma unroll
        for (int i = 0; i < 8; ++i) ss += y[i] * y[i];
        const float r = rsqrtf(row_sum<D>(ss) * (1.f / D) + a.eps);
#pragma unroll
        for (int i = 0; i < 8; ++i) y[i] = y[i] * r * (is_k ? wk[i] : wq[i]);
        turn<false>(tn, a.interleaved, y);
        if (h >= n_rows) continue;
        __nv_bfloat16* to;
        if (!is_k) to = a.q_out + ((int64_t)t * a.Hq + h) * D;
        else if constexpr (kStore) to = kv_row ? kv_row + (int64_t)(h - a.Hq) * a.P * D : nullptr;
        else to = a.k_out + ((int64_t)t * a.Hkv + h - a.Hq) * D;
        if (to) *reinterpret_cast<uint4*>(to + e0) = is_v ? raw[u] : pack8(y);
    }
}

// Backwards.  A CTA's warps take tasks (a token's kTaskRows query or key rows) in
// turn and add up the weights' gradients of their lanes' elements; the CTA's sums
// go to one partial row, added by a second kernel in a fixed order.
template <int D>
__global__ void __launch_bounds__(kNormThreads)
    sq_norm_rope_grad_kernel(const __grid_constant__ NormRopeGradArgs a) {
    using C = NormCfg<D>;
    grid_dependency_wait();
    grid_launch_dependents();
    constexpr int kWarps = kNormThreads / 32;
    __shared__ float red[kWarps][2][D];
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int sub = lane / C::kLanes, e0 = (lane % C::kLanes) * 8;
    const int n_rows = a.Hq + a.Hkv;
    const unsigned chunks = (unsigned)(n_rows + C::kTaskRows - 1) / C::kTaskRows;
    const unsigned tasks = (unsigned)a.n * chunks;
    float wq[8], wk[8], gq[8], gk[8];
    load_weights(a.q_weight, a.weight_f32, e0, wq);
    load_weights(a.k_weight, a.weight_f32, e0, wk);
#pragma unroll
    for (int i = 0; i < 8; ++i) gq[i] = gk[i] = 0.f;
    for (unsigned task = blockIdx.x * kWarps + warp; task < tasks; task += gridDim.x * kWarps) {
        const unsigned t = task / chunks;
        const int row0 = (int)(task - t * chunks) * C::kTaskRows + sub;
        uint4 rx[kUnroll], rz[kUnroll];
#pragma unroll
        for (int u = 0; u < kUnroll; ++u) {
            const int h = row0 + u * C::kGroups;
            const bool is_k = h >= a.Hq;
            rx[u] = rz[u] = make_uint4(0, 0, 0, 0);
            if (h < n_rows) {
                rx[u] = ld_row((is_k ? a.k + t * a.k_stride + (int64_t)(h - a.Hq) * D
                                     : a.q + t * a.q_stride + (int64_t)h * D) + e0);
                rz[u] = ld_row((is_k ? a.dk_out + ((int64_t)t * a.Hkv + h - a.Hq) * D
                                     : a.dq_out + ((int64_t)t * a.Hq + h) * D) + e0);
            }
        }
        Turn tn;
        int pos = a.positions ? __ldg(&a.positions[t]) : 0;
        if (a.rot > 0) pos = checked_pos(pos, a.max_pos, a.err);
        load_turn(tn, a.rope, pos, a.rot, a.interleaved, e0, sub * C::kLanes);
#pragma unroll
        for (int u = 0; u < kUnroll; ++u) {
            const int h = row0 + u * C::kGroups;
            if (row0 - sub + u * C::kGroups >= n_rows) break;  // (warp-uniform)
            const bool is_k = h >= a.Hq;
            float x[8], dy[8];
            unpack8(rx[u], x);
            unpack8(rz[u], dy);
            turn<true>(tn, a.interleaved, dy);
            float ss = 0.f;
#pragma unroll
            for (int i = 0; i < 8; ++i) ss += x[i] * x[i];
            // (rows past the token's heads add nothing)
            const float rs = rsqrtf(row_sum<D>(ss) * (1.f / D) + a.eps);
            const float r = h < n_rows ? rs : 0.f;
            float dot = 0.f;
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                x[i] *= r;
                const float g = dy[i] * x[i];
                if (is_k) gk[i] += g;
                else gq[i] += g;
                dy[i] *= is_k ? wk[i] : wq[i];
                dot += dy[i] * x[i];
            }
            dot = row_sum<D>(dot) * (1.f / D);
#pragma unroll
            for (int i = 0; i < 8; ++i) dy[i] = r * (dy[i] - x[i] * dot);
            if (h < n_rows)
                *reinterpret_cast<uint4*>((is_k ? a.dk + t * a.dk_stride + (int64_t)(h - a.Hq) * D
                                                : a.dq + t * a.dq_stride + (int64_t)h * D) + e0) =
                    pack8(dy);
        }
    }
    if (!a.part) return;
    // the lane groups of the warp, then the warps
#pragma unroll
    for (int o = C::kLanes; o < 32; o <<= 1)
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            gq[i] += __shfl_xor_sync(0xffffffffu, gq[i], o);
            gk[i] += __shfl_xor_sync(0xffffffffu, gk[i], o);
        }
    if (sub == 0) {
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            red[warp][0][e0 + i] = gq[i];
            red[warp][1][e0 + i] = gk[i];
        }
    }
    __syncthreads();
    for (int i = threadIdx.x; i < 2 * D; i += kNormThreads) {
        float s = 0.f;
#pragma unroll
        for (int w = 0; w < kWarps; ++w) s += (&red[w][0][0])[i];
        a.part[(size_t)blockIdx.x * 2 * D + i] = s;
    }
}

// Adds the CTAs' partial gradients: 32 columns a block, 32 threads a column.
template <int D>
__global__ void __launch_bounds__(1024)
    sq_norm_rope_grad_sum_kernel(const float* part, int ctas, float* dq_weight, float* dk_weight) {
    grid_dependency_wait();
    grid_launch_dependents();
    __shared__ float red[32][33];
    const int x = threadIdx.x & 31, y = threadIdx.x >> 5;
    const int col = blockIdx.x * 32 + x;
    float s = 0.f;
    for (int c = y; c < ctas; c += 32) s += part[(size_t)c * 2 * D + col];
    red[y][x] = s;
    __syncthreads();
    // warp y now adds column y
    s = red[x][y];
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) s += __shfl_xor_sync(0xffffffffu, s, o);
    const int out = blockIdx.x * 32 + y;
    float* to = out < D ? dq_weight : dk_weight;
    if (x == 0 && to) to[out < D ? out : out - D] = s;
}

template <typename... P, typename... A>
cudaError_t launch_after(void (*kernel)(P...), unsigned grid, unsigned block, cudaStream_t st, A... args) {
    cudaLaunchAttribute at;
    at.id = cudaLaunchAttributeProgrammaticStreamSerialization;
    at.val.programmaticStreamSerializationAllowed = 1;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3(grid);
    cfg.blockDim = dim3(block);
    cfg.stream = st;
    cfg.attrs = &at;
    cfg.numAttrs = 1;
    return cudaLaunchKernelEx(&cfg, kernel, args...);
}

template <int D, bool kStore, typename Args>
cudaError_t launch_rows(const Args& a, cudaStream_t st) {
    const int rows = a.Hq + (kStore ? 2 : 1) * a.Hkv;
    const int64_t warps = (int64_t)a.n * ((rows + NormCfg<D>::kTaskRows - 1) / NormCfg<D>::kTaskRows);
    if (warps == 0) return cudaSuccess;
    constexpr int per = kNormThreads / 32;
    return launch_after(sq_norm_rope_kernel<D, kStore, Args>, (unsigned)((warps + per - 1) / per),
                        kNormThreads, st, a);
}

template <int D>
cudaError_t launch_grad(const NormRopeGradArgs& a, cudaStream_t st) {
    cudaError_t e = launch_after(sq_norm_rope_grad_kernel<D>, (unsigned)a.ctas, kNormThreads, st, a);
    if (e != cudaSuccess || !a.part) return e;
    return launch_after(sq_norm_rope_grad_sum_kernel<D>, 2 * D / 32, 1024, st, (const float*)a.part,
                        (int)a.ctas, a.dq_weight, a.dk_weight);
}

}  // namespace

cudaError_t launch_norm_rope(const NormRopeArgs& a, int D, bool store, cudaStream_t st) {
    if (D == 128) return store ? launch_rows<128, true>(a, st) : launch_rows<128, false>(a, st);
    return store ? launch_rows<64, true>(a, st) : launch_rows<64, false>(a, st);
}

cudaError_t launch_norm_rope_inline(const NormRopeInlineArgs& a, int D, cudaStream_t st) {
    return D == 128 ? launch_rows<128, true>(a, st) : launch_rows<64, true>(a, st);
}

int norm_rope_grad_ctas(int32_t n, int32_t heads, int D, int num_sms) {
    const int task = D == 128 ? NormCfg<128>::kTaskRows : NormCfg<64>::kTaskRows;
    const int64_t tasks = (int64_t)n * ((heads + task - 1) / task);
    constexpr int per = kNormThreads / 32;
    return (int)std::max<int64_t>(1, std::min<int64_t>((tasks + per - 1) / per, 3 * (int64_t)num_sms));
}

cudaError_t launch_norm_rope_grad(const NormRopeGradArgs& a, int D, cudaStream_t st) {
    return D == 128 ? launch_grad<128>(a, st) : launch_grad<64>(a, st);
}

}  // namespace sq
