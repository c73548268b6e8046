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
// way.  To keep the SMs' issue slots out of the way a lane holds both halves of
// its pairs: D / 8 lanes take a row, each four elements f .. f + 3 and the four
// g .. g + 3 they turn with, so that the rotation needs no shuffle; the weight and
// the cosine are one factor of each element, made once for a warp's rows; and the
// products go two at a time (fma.rn.f32x2).  A warp's task is up to kUnroll rows
// of each of its lane groups, all query, all key or all value heads of one token:
// its loads are all issued before the first is used.
#include <algorithm>
#include <type_traits>

#include "norm_rope.cuh"

namespace sq {
namespace {

using namespace dev;

constexpr int kNormThreads = 128;
constexpr int kUnroll = 8;      // rows of a lane group in flight
constexpr int kGradThreads = 256;
constexpr int kGradUnroll = 4;  // ... backwards, of two tensors

// Tasks of a token: its query heads, its key heads, its value heads (kStore).
template <int D, int kRows>
struct Tasks {
    int q, k, total;
    __host__ __device__ Tasks(int Hq, int Hkv, bool store) {
        constexpr int n = NormCfg<D>::kGroups * kRows;
        q = (Hq + n - 1) / n;
        k = (Hkv + n - 1) / n;
        total = q + k + (store ? k : 0);
    }
};

// What is left to gain is the memory's: with 28 warps an SM (72 registers a thread, 12
// to 52 bytes of them spilled) 12,982 tokens of 32 query and 8 key heads of 128,
// stored, take 57.3 us, 5.6 TB/s (24 warps 60, 32 warps, with more spills, 57.5 where
// these took 56.7; a warp that takes a token's tasks in turn, the next one's rows
// loaded ahead, in 16 warps 64).
template <int D, bool kStore, bool kPairs, typename Args>
__global__ void __launch_bounds__(kNormThreads, 7)
    sq_norm_rope_kernel(const __grid_constant__ Args a) {
    using C = NormCfg<D>;
    constexpr bool kInline = std::is_same<Args, NormRopeInlineArgs>::value;
    grid_dependency_wait();
    grid_launch_dependents();
    const int lane = threadIdx.x & 31;
    const Tasks<D, kUnroll> per(a.Hq, a.Hkv, kStore);
    // (n x tasks fits: the rows of as many tokens would not fit the device)
    const unsigned task = blockIdx.x * (kNormThreads / 32) + (threadIdx.x >> 5);
    const unsigned t = task / (unsigned)per.total;
    if (t >= (unsigned)a.n) return;
    int part = (int)(task - t * per.total);
    const bool is_v = part >= per.q + per.k, is_k = part >= per.q;
    if (is_k) part -= per.q;
    if (is_v) part -= per.k;
    const int sub = lane / C::kLanes, l = lane % C::kLanes;
    const int heads = is_k ? a.Hkv : a.Hq;
    const int h0 = part * C::kGroups * kUnroll;   // first head of the warp's
    const int n_pass = min(kUnroll, (heads - h0 + C::kGroups - 1) / C::kGroups);
    const int h = h0 + sub;
    const __nv_bfloat16* src = (is_v ? a.v + t * a.v_stride : is_k ? a.k + t * a.k_stride : a.q + t * a.q_stride) +
                               (int64_t)h * D;
    RowPlace place = {0, 0};
    if constexpr (kStore) {
        if constexpr (kInline) place = a.inline_place[t];
        else place = a.places[t];
    }
    // where head h goes, and the elements from head to head
    __nv_bfloat16* dst = nullptr;
    int64_t step = D;
    if (!is_k) {
        dst = a.q_out + ((int64_t)t * a.Hq + h) * D;
    } else if constexpr (kStore) {
        const int lp = __ffs(a.P) - 1;
        const int64_t page = place.row >> lp;
        step = (int64_t)a.P * D;
        if (place.row >= 0 && page < a.num_pages)
            dst = a.pool + ((((int64_t)a.layer * a.num_pages + page) * 2 + (is_v ? 1 : 0)) * a.Hkv + h) * step +
                  (int64_t)(place.row & (a.P - 1)) * D;
        else set_error(a.err, kErrBounds);
    } else {
        dst = a.k_out + ((int64_t)t * a.Hkv + h) * D;
    }
    if (kStore && is_v) {
        uint4 raw[kUnroll];
#pragma unroll
        for (int u = 0; u < kUnroll; ++u)
            if (h + u * C::kGroups < heads) raw[u] = ld_row(src + u * C::kGroups * D + 8 * l);
#pragma unroll
        for (int u = 0; u < kUnroll; ++u)
            if (h + u * C::kGroups < heads && dst)
                *reinterpret_cast<uint4*>(dst + u * C::kGroups * step + 8 * l) = raw[u];
        return;
    }
    Lane ln;
    ln.init<kPairs>(l, a.rot);
    uint2 rf[kUnroll], rg[kUnroll];
#pragma unroll
    for (int u = 0; u < kUnroll; ++u) {
        rf[u] = rg[u] = make_uint2(0, 0);
        if (h + u * C::kGroups < heads) {
            rf[u] = ld_half_row(src + u * C::kGroups * D + ln.f);
            rg[u] = ld_half_row(src + u * C::kGroups * D + ln.g);
        }
    }
    // out = r (x A + other B): A the weight times the cosine, B the other's weight
    // times the sine
    f32x2 A[4], B[4];
    {
        Turn tn;
        int pos = a.positions ? __ldg(&a.positions[t]) : place.pos;
        if (a.rot > 0) pos = checked_pos(pos, a.max_pos, a.err);
        load_turn<kPairs>(tn, a.rope, pos, a.rot, ln);
        Eight w;
        load_weights(is_k ? a.k_weight : a.q_weight, a.weight_f32, ln, w);
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            A[i] = mul2(w.v[i], tn.c[i]);
            B[i] = mul2(w.other<kPairs>(i), tn.s[i]);
        }
    }
#pragma unroll
    for (int u = 0; u < kUnroll; ++u) {
        if (u >= n_pass) break;  // (warp-uniform)
        Eight x;
        x.set(rf[u], rg[u]);
        f32x2 ss = mul2(x.v[0], x.v[0]);
#pragma unroll
        for (int i = 1; i < 4; ++i) ss = fma2(x.v[i], x.v[i], ss);
        const float r = rsqrtf(row_sum<D>(ss) * (1.f / D) + a.eps);
        const f32x2 rr = f2(r, r);
        uint32_t o[4];
#pragma unroll
        for (int i = 0; i < 4; ++i)
            o[i] = pack2(mul2(fma2(x.v[i], A[i], ln.turned(mul2(x.other<kPairs>(i), B[i]))), rr));
        if (h + u * C::kGroups < heads && dst) {
            __nv_bfloat16* to = dst + u * C::kGroups * step;
            *reinterpret_cast<uint2*>(to + ln.f) = make_uint2(o[0], o[1]);
            *reinterpret_cast<uint2*>(to + ln.g) = make_uint2(o[2], o[3]);
        }
    }
}

// Backwards.  A CTA's warps take tasks (query or key heads of a token) in turn and
// add up the weights' gradients of their lanes' elements; the CTA's sums go to one
// partial row, added by a second kernel in a fixed order.  8,192 tokens of 64 query
// and 8 key heads of 128: 85 us, 5.3 TB/s (before the elements that do not turn were
// kept apart 84; then two rows of a lane group in flight 103, eight 105, a position
// read a task ahead 86, the next task's rows copied into shared memory ahead 85).
template <int D, bool kPairs>
__global__ void __launch_bounds__(kGradThreads)
    sq_norm_rope_grad_kernel(const __grid_constant__ NormRopeGradArgs a) {
    using C = NormCfg<D>;
    grid_dependency_wait();
    grid_launch_dependents();
    constexpr int kWarps = kGradThreads / 32;
    __shared__ float red[kWarps][2][D];
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int sub = lane / C::kLanes;
    const Tasks<D, kGradUnroll> per(a.Hq, a.Hkv, false);
    const unsigned tasks = (unsigned)a.n * per.total;
    Lane ln;
    ln.init<kPairs>(lane % C::kLanes, a.rot);
    Eight wq, wk;
    load_weights(a.q_weight, a.weight_f32, ln, wq);
    load_weights(a.k_weight, a.weight_f32, ln, wk);
    f32x2 gq[4], gk[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) gq[i] = gk[i] = f2(0.f, 0.f);
    for (unsigned task = blockIdx.x * kWarps + warp; task < tasks; task += gridDim.x * kWarps) {
        const unsigned t = task / (unsigned)per.total;
        int part = (int)(task - t * per.total);
        const bool is_k = part >= per.q;
        if (is_k) part -= per.q;
        const int heads = is_k ? a.Hkv : a.Hq;
        const int h0 = part * C::kGroups * kGradUnroll, h = h0 + sub;
        const int n_pass = min(kGradUnroll, (heads - h0 + C::kGroups - 1) / C::kGroups);
        const __nv_bfloat16* xs = (is_k ? a.k + t * a.k_stride : a.q + t * a.q_stride) + (int64_t)h * D;
        const __nv_bfloat16* zs = (is_k ? a.dk_out : a.dq_out) + ((int64_t)t * heads + h) * D;
        __nv_bfloat16* dst = (is_k ? a.dk + t * a.dk_stride : a.dq + t * a.dq_stride) + (int64_t)h * D;
        uint2 xf[kGradUnroll], xg[kGradUnroll], zf[kGradUnroll], zg[kGradUnroll];
#pragma unroll
        for (int u = 0; u < kGradUnroll; ++u) {
            xf[u] = xg[u] = zf[u] = zg[u] = make_uint2(0, 0);
            if (h + u * C::kGroups < heads) {
                xf[u] = ld_half_row(xs + u * C::kGroups * D + ln.f);
                xg[u] = ld_half_row(xs + u * C::kGroups * D + ln.g);
                zf[u] = ld_half_row(zs + u * C::kGroups * D + ln.f);
                zg[u] = ld_half_row(zs + u * C::kGroups * D + ln.g);
            }
        }
        Turn tn;
        int pos = a.positions ? __ldg(&a.positions[t]) : 0;
        if (a.rot > 0) pos = checked_pos(pos, a.max_pos, a.err);
        load_turn<kPairs>(tn, a.rope, pos, a.rot, ln);
#pragma unroll
        for (int u = 0; u < kGradUnroll; ++u) {
            if (u >= n_pass) break;  // (warp-uniform)
            Eight x, z;
            x.set(xf[u], xg[u]);
            z.set(zf[u], zg[u]);
            f32x2 ss = mul2(x.v[0], x.v[0]);
#pragma unroll
            for (int i = 1; i < 4; ++i) ss = fma2(x.v[i], x.v[i], ss);
            const float rs = rsqrtf(row_sum<D>(ss) * (1.f / D) + a.eps);
            // (rows past the token's heads add nothing)
            const float r = h + u * C::kGroups < heads ? rs : 0.f;
            const f32x2 rr = f2(r, r), back = f2(-1.f, -1.f);
            f32x2 dn[4], dot = f2(0.f, 0.f);
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                // dy: dz turned back
                const f32x2 dy = fma2(z.v[i], tn.c[i], ln.turned(mul2(mul2(z.other<kPairs>(i), tn.s[i]), back)));
                x.v[i] = mul2(x.v[i], rr);
                if (is_k) gk[i] = fma2(dy, x.v[i], gk[i]);
                else gq[i] = fma2(dy, x.v[i], gq[i]);
                dn[i] = mul2(dy, is_k ? wk.v[i] : wq.v[i]);
                dot = fma2(dn[i], x.v[i], dot);
            }
            const float m = row_sum<D>(dot) * (-1.f / D);
            const f32x2 mm = f2(m, m);
            uint32_t o[4];
#pragma unroll
            for (int i = 0; i < 4; ++i) o[i] = pack2(mul2(fma2(x.v[i], mm, dn[i]), rr));
            if (h + u * C::kGroups < heads) {
                __nv_bfloat16* to = dst + u * C::kGroups * D;
                *reinterpret_cast<uint2*>(to + ln.f) = make_uint2(o[0], o[1]);
                *reinterpret_cast<uint2*>(to + ln.g) = make_uint2(o[2], o[3]);
            }
        }
    }
    if (!a.part) return;
    // the lane groups of the warp, then the warps
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        float2 q = un2(gq[i]), k = un2(gk[i]);
#pragma unroll
        for (int o = C::kLanes; o < 32; o <<= 1) {
            q.x += __shfl_xor_sync(0xffffffffu, q.x, o);
            q.y += __shfl_xor_sync(0xffffffffu, q.y, o);
            k.x += __shfl_xor_sync(0xffffffffu, k.x, o);
            k.y += __shfl_xor_sync(0xffffffffu, k.y, o);
        }
        if (sub == 0) {
            const int e = (i < 2 ? ln.f : ln.g) + 2 * (i & 1);
            red[warp][0][e] = q.x;
            red[warp][0][e + 1] = q.y;
            red[warp][1][e] = k.x;
            red[warp][1][e + 1] = k.y;
        }
    }
    __syncthreads();
    for (int i = threadIdx.x; i < 2 * D; i += kGradThreads) {
        float s = 0.f;
#pragma unroll
        for (int w = 0; w < kWarps; ++w) s += (&red[w][0][0])[i];
        a.part[(size_t)blockIdx.x * 2 * D + i] = s;
    }
}

// Adds the CTAs' partial gradients: eight columns a block, 128 threads a column.
constexpr int kSumCols = 8;
template <int D>
__global__ void __launch_bounds__(1024)
    sq_norm_rope_grad_sum_kernel(const float* part, int ctas, float* dq_weight, float* dk_weight) {
    grid_dependency_wait();
    grid_launch_dependents();
    __shared__ float red[128][kSumCols + 1];
    const int x = threadIdx.x % kSumCols, y = threadIdx.x / kSumCols;
    const int col0 = blockIdx.x * kSumCols;
    float s = 0.f;
#pragma unroll 4
    for (int c = y; c < ctas; c += 128) s += part[(size_t)c * 2 * D + col0 + x];
    red[y][x] = s;
    __syncthreads();
    // the first warps add a column each
    const int w = threadIdx.x >> 5, lane = threadIdx.x & 31;
    if (w >= kSumCols) return;
    s = (red[lane][w] + red[lane + 32][w]) + (red[lane + 64][w] + red[lane + 96][w]);
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) s += __shfl_xor_sync(0xffffffffu, s, o);
    const int out = col0 + w;
    float* to = out < D ? dq_weight : dk_weight;
    if (lane == 0 && to) to[out < D ? out : out - D] = s;
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
    const int64_t warps = (int64_t)a.n * Tasks<D, kUnroll>(a.Hq, a.Hkv, kStore).total;
    if (warps == 0) return cudaSuccess;
    constexpr int per = kNormThreads / 32;
    const unsigned grid = (unsigned)((warps + per - 1) / per);
    return a.interleaved ? launch_after(sq_norm_rope_kernel<D, kStore, true, Args>, grid, kNormThreads, st, a)
                         : launch_after(sq_norm_rope_kernel<D, kStore, false, Args>, grid, kNormThreads, st, a);
}

template <int D>
cudaError_t launch_grad(const NormRopeGradArgs& a, cudaStream_t st) {
    const cudaError_t e =
        a.interleaved ? launch_after(sq_norm_rope_grad_kernel<D, true>, (unsigned)a.ctas, kGradThreads, st, a)
                      : launch_after(sq_norm_rope_grad_kernel<D, false>, (unsigned)a.ctas, kGradThreads, st, a);
    if (e != cudaSuccess || !a.part) return e;
    return launch_after(sq_norm_rope_grad_sum_kernel<D>, 2 * D / kSumCols, 1024, st, (const float*)a.part,
                        (int)a.ctas, a.dq_weight, a.dk_weight);
}

template <int D>
int grad_ctas(int32_t n, int32_t Hq, int32_t Hkv, int num_sms) {
    const int64_t tasks = (int64_t)n * Tasks<D, kGradUnroll>(Hq, Hkv, false).total;
    constexpr int per = kGradThreads / 32;
    return (int)std::max<int64_t>(1, std::min<int64_t>((tasks + per - 1) / per, 2 * (int64_t)num_sms));
}

}  // namespace

cudaError_t launch_norm_rope(const NormRopeArgs& a, int D, bool store, cudaStream_t st) {
    if (D == 128) return store ? launch_rows<128, true>(a, st) : launch_rows<128, false>(a, st);
    return store ? launch_rows<64, true>(a, st) : launch_rows<64, false>(a, st);
}

cudaError_t launch_norm_rope_inline(const NormRopeInlineArgs& a, int D, cudaStream_t st) {
    return D == 128 ? launch_rows<128, true>(a, st) : launch_rows<64, true>(a, st);
}

int norm_rope_grad_ctas(int32_t n, int32_t Hq, int32_t Hkv, int D, int num_sms) {
    return D == 128 ? grad_ctas<128>(n, Hq, Hkv, num_sms) : grad_ctas<64>(n, Hq, Hkv, num_sms);
}

cudaError_t launch_norm_rope_grad(const NormRopeGradArgs& a, int D, cudaStream_t st) {
    return D == 128 ? launch_grad<128>(a, st) : launch_grad<64>(a, st);
}

}  // namespace sq
