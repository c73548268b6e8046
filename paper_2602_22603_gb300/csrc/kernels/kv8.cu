// Rows of a cache held in 8 bits: stored (with the norms and the rotation on the
// way), copied on write, read back, and compacted after an eviction.
//
// A block is kScaleRows slots of one page, plane and head, and has one scale s = 2^e;
// an element x of it is held as the e4m3 code of x / s, so that
//     e = max(kLeastScale, ceil(log2(max |x| / 448))),   x ~ code * s.
// e4m3 has 4 significant bits at any size down to 2^-6, and a power of two moves
// sizes alone: the values that a block stands for do not depend on its scale but
// where they are below 2^-6 s, 2^-13 of the block's largest or less.  So rows may be
// taken from scale to scale (a new row in a block that has rows, rows of several
// blocks packed into one) without their errors adding up.
#include <algorithm>
#include <type_traits>

#include "e4m3.cuh"
#include "norm_rope.cuh"

namespace sq {
namespace {

using namespace dev;

constexpr int kStoreThreads = 128;
constexpr int kHeadRows = 8;   // query rows of a lane group in flight

__device__ __forceinline__ int log2_of(int power) { return __ffs(power) - 1; }

// Offset of a plane's first row in the codes, in rows.
__device__ __forceinline__ int64_t plane_row(const Kv8Pool& p, int layer, int64_t page, int kv, int head) {
    return (((layer * p.num_pages + page) * 2 + kv) * p.Hkv + head) * p.P;
}

// Tasks of a block of a run: its keys' and its values' heads, then the query heads of
// `most` rows.
template <int D>
struct StoreTasks {
    int q, total;
    __host__ __device__ StoreTasks(int Hq, int Hkv, int most) {
        constexpr int n = NormCfg<D>::kGroups * kHeadRows;
        q = (Hq + n - 1) / n;
        total = 2 * Hkv + most * q;
    }
};

// A warp to a block of keys or values (the rows it has before the run's first are
// read, and written again where the scale changes), or to the query rows of up to
// kHeadRows heads of each lane group of a token.  Its bytes bound it, less directly its
// issue slots (59% of them): 13,015 rows of three prompts, 32/8 heads of 128 dimensions,
// 293 MB in 57.5 us (0.75 of the copy peak).  Rows of 4 heads in flight take 76 us, of 16
// 58 .. 64, a CTA of 64 threads 64; more warps an SM (64 registers) change nothing.
template <int D, bool kPairs>
__global__ void __launch_bounds__(kStoreThreads)
    sq_kv8_store_kernel(const __grid_constant__ Kv8StoreInlineArgs a) {
    using C = NormCfg<D>;
    grid_dependency_wait();
    grid_launch_dependents();
    const int lane = threadIdx.x & 31;
    const StoreTasks<D> per(a.Hq, a.Hkv, a.most);
    const unsigned task = blockIdx.x * (kStoreThreads / 32) + (threadIdx.x >> 5);
    const unsigned at = task / (unsigned)per.total, r = at / (unsigned)a.blocks;
    if (r >= (unsigned)a.n_runs) return;
    int part = (int)(task - at * per.total);
    RowRun run = a.runs ? a.runs[r] : a.inline_run[r];
    {
        // the block's rows of it
        const int b0 = (run.row & ~(kScaleRows - 1)) + (int)(at - r * a.blocks) * kScaleRows;
        const int from = max(run.row, b0), skip = from - run.row;
        run.n = min(run.row + run.n, b0 + kScaleRows) - from;
        if (run.n <= 0) return;
        run.row = from;
        run.first += skip;
        run.pos += skip;
    }
    const int sub = lane / C::kLanes, l = lane % C::kLanes;
    Lane ln;
    if (part >= 2 * a.Hkv) {
        part -= 2 * a.Hkv;
        const int i = part / per.q;
        if (i >= run.n) return;
        const int64_t t = run.first + i;
        const int h0 = (part - i * per.q) * C::kGroups * kHeadRows, h = h0 + sub;
        const int n_pass = min(kHeadRows, (a.Hq - h0 + C::kGroups - 1) / C::kGroups);
        ln.init<kPairs>(l, a.rot);
        const __nv_bfloat16* src = a.q + t * a.q_stride + (int64_t)h * D;
        __nv_bfloat16* dst = a.q_out + (t * a.Hq + h) * D;
        uint2 rf[kHeadRows], rg[kHeadRows];
#pragma unroll
        for (int u = 0; u < kHeadRows; ++u) {
            rf[u] = rg[u] = make_uint2(0, 0);
            if (h + u * C::kGroups < a.Hq) {
                rf[u] = ld_half_row(src + u * C::kGroups * D + ln.f);
                rg[u] = ld_half_row(src + u * C::kGroups * D + ln.g);
            }
        }
        Turn tn;
        int pos = a.positions ? __ldg(&a.positions[t]) : run.pos + i;
        if (a.rot > 0) pos = checked_pos(pos, a.max_pos, a.err);
        load_turn<kPairs>(tn, a.rope, pos, a.rot, ln);
        Eight w;
        load_weights(a.q_weight, a.weight_f32, ln, w);
        f32x2 A[4], B[4];
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            A[k] = mul2(w.v[k], tn.c[k]);
            B[k] = mul2(w.other<kPairs>(k), tn.s[k]);
        }
#pragma unroll
        for (int u = 0; u < kHeadRows; ++u) {
            if (u >= n_pass) break;  // (warp-uniform)
            Eight x;
            x.set(rf[u], rg[u]);
            f32x2 ss = mul2(x.v[0], x.v[0]);
#pragma unroll
            for (int k = 1; k < 4; ++k) ss = fma2(x.v[k], x.v[k], ss);
            const float rs = rsqrtf(row_sum<D>(ss) * (1.f / D) + a.eps);
            const f32x2 rr = f2(rs, rs);
            uint32_t o[4];
#pragma unroll
            for (int k = 0; k < 4; ++k)
                o[k] = pack2(mul2(fma2(x.v[k], A[k], ln.turned(mul2(x.other<kPairs>(k), B[k]))), rr));
            if (h + u * C::kGroups < a.Hq) {
                __nv_bfloat16* to = dst + u * C::kGroups * D;
                *reinterpret_cast<uint2*>(to + ln.f) = make_uint2(o[0], o[1]);
                *reinterpret_cast<uint2*>(to + ln.g) = make_uint2(o[2], o[3]);
            }
        }
        return;
    }
    const bool is_v = part >= a.Hkv;
    const int head = is_v ? part - a.Hkv : part;
    const bool norm = !is_v && !a.plain;
    const int lp = log2_of(a.pool.P);
    const int64_t page = run.row >> lp;
    const int s0 = run.row & (kScaleRows - 1), s1 = s0 + run.n;
    if (run.row < 0 || page >= a.pool.num_pages || s1 > kScaleRows) {
        if (lane == 0) set_error(a.err, kErrBounds);
        return;
    }
    const int64_t row0 = plane_row(a.pool, a.layer + blockIdx.y, page, is_v, head) +
                         ((run.row & (a.pool.P - 1)) - s0);
    uint8_t* codes = a.pool.codes + row0 * D;
    float* scale = a.pool.scales + row0 / kScaleRows;
    const int64_t stride = is_v ? a.v_stride : a.k_stride;
    const __nv_bfloat16* src = (is_v ? a.v : a.k) + blockIdx.y * a.layer_stride + run.first * stride + head * D;
    ln.init<kPairs>(l, norm ? a.rot : 0);
    constexpr int kPass = kScaleRows / C::kGroups;
    // raw: a new row's 16 bytes of this lane, or 8 codes of one that is there
    uint2 rf[kPass], rg[kPass];
#pragma unroll
    for (int u = 0; u < kPass; ++u) {
        const int i = u * C::kGroups + sub;
        rf[u] = rg[u] = make_uint2(0, 0);
        if (i >= s0 && i < s1) {
            rf[u] = ld_half_row(src + (i - s0) * stride + ln.f);
            rg[u] = ld_half_row(src + (i - s0) * stride + ln.g);
        } else if (i < s0) {
            rf[u].x = *reinterpret_cast<const uint32_t*>(codes + i * D + ln.f);
            rg[u].x = *reinterpret_cast<const uint32_t*>(codes + i * D + ln.g);
        }
    }
    const float old = s0 > 0 ? *scale : 0.f;
    Eight w;
    if (norm) load_weights(a.k_weight, a.weight_f32, ln, w);
    // (rows that are none are zeros)
    Eight x[kPass];
#pragma unroll
    for (int u = 0; u < kPass; ++u) {
        const int i = u * C::kGroups + sub;
        x[u].set(rf[u], rg[u]);
        if (norm) {
            // (every lane: the sums are the warp's)
            Turn tn;
            int pos = 0;
            if (i >= s0 && i < s1) {
                pos = a.positions ? __ldg(&a.positions[run.first + i - s0]) : run.pos + i - s0;
                if (a.rot > 0) pos = checked_pos(pos, a.max_pos, a.err);
            }
            load_turn<kPairs>(tn, a.rope, pos, a.rot, ln);
            f32x2 ss = mul2(x[u].v[0], x[u].v[0]);
#pragma unroll
            for (int k = 1; k < 4; ++k) ss = fma2(x[u].v[k], x[u].v[k], ss);
            const float rs = rsqrtf(row_sum<D>(ss) * (1.f / D) + a.eps);
            const f32x2 rr = f2(rs, rs);
            Eight y;
#pragma unroll
            for (int k = 0; k < 4; ++k)
                y.v[k] = mul2(fma2(x[u].v[k], mul2(w.v[k], tn.c[k]),
                                   ln.turned(mul2(x[u].other<kPairs>(k), mul2(w.other<kPairs>(k), tn.s[k])))),
                              rr);
            x[u] = y;
        }
        if (i < s0) {
            const float4 f = e4m3_values(rf[u].x, old), g = e4m3_values(rg[u].x, old);
            x[u].v[0] = f2(f.x, f.y);
            x[u].v[1] = f2(f.z, f.w);
            x[u].v[2] = f2(g.x, g.y);
            x[u].v[3] = f2(g.z, g.w);
        }
        if (i >= s1) x[u].v[0] = x[u].v[1] = x[u].v[2] = x[u].v[3] = 0;
    }
    // the largest size (NaN is none; an infinity, seldom, is left out the second time)
    float size = 0.f;
#pragma unroll
    for (int u = 0; u < kPass; ++u)
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            const float2 v = un2(x[u].v[k]);
            size = fmaxf(fmaxf(fabsf(v.x), fabsf(v.y)), size);
        }
    size = warp_size(size);
    const bool odd = !(size < 0x1.fp127f);   // (and sizes that round to infinities)
    if (odd) {
        size = 0.f;
#pragma unroll
        for (int u = 0; u < kPass; ++u)
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                const float2 v = un2(x[u].v[k]);
                size = fmaxf(fmaxf(finite_size(v.x), finite_size(v.y)), size);
            }
        size = warp_size(size);
    }
    const int e = scale_exponent(size);
    const float s = power_of_two(e);
    const f32x2 inv = f2(power_of_two(-e), power_of_two(-e));
#pragma unroll
    for (int u = 0; u < kPass; ++u) {
        const int i = u * C::kGroups + sub;
        if (i >= s1 || (i < s0 && s == old)) continue;
        uint32_t c[4];
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            const float2 v = un2(mul2(x[u].v[k], inv));
            c[k] = odd ? to_e4m3x2(v.x, v.y, e < kMostScale ? 448.f : 240.f) : to_e4m3x2(v.x, v.y);
        }
        *reinterpret_cast<uint32_t*>(codes + i * D + ln.f) = c[0] | c[1] << 16;
        *reinterpret_cast<uint32_t*>(codes + i * D + ln.g) = c[2] | c[3] << 16;
    }
    if (lane == 0) *scale = s;
}

// ---- copies of pages' first rows (copy-on-write) --------------------------------
constexpr int kCopyThreads = 128;

// A CTA to a page's rows of one plane and head; the launch also takes the row limits of
// plans that the longer sequences leave valid.
__global__ void __launch_bounds__(kCopyThreads)
    sq_kv8_copy_kernel(const __grid_constant__ Kv8CopyArgs a, int D) {
    grid_dependency_wait();
    grid_launch_dependents();
    if (blockIdx.x == 0 && threadIdx.x < a.lens.n) *a.lens.ptr[threadIdx.x] = a.lens.val[threadIdx.x];
    const int planes = a.L * 2 * a.pool.Hkv;
    const int copy = blockIdx.x / planes, plane = blockIdx.x % planes;
    if (copy >= a.n_cow) return;
    const CowCopy c = a.cow[copy];
    if ((uint64_t)c.src_page >= (uint64_t)a.pool.num_pages || (uint64_t)c.dst_page >= (uint64_t)a.pool.num_pages ||
        c.rows < 0 || c.rows > a.pool.P) {
        if (threadIdx.x == 0) set_error(a.err, kErrBounds);
        return;
    }
    const int head = plane % a.pool.Hkv, kv = plane / a.pool.Hkv % 2, layer = plane / (2 * a.pool.Hkv);
    const int64_t from = plane_row(a.pool, layer, c.src_page, kv, head);
    const int64_t to = plane_row(a.pool, layer, c.dst_page, kv, head);
    const uint4* x = reinterpret_cast<const uint4*>(a.pool.codes + from * D);
    uint4* y = reinterpret_cast<uint4*>(a.pool.codes + to * D);
    for (int i = threadIdx.x; i < c.rows * (D / 16); i += kCopyThreads) y[i] = x[i];
    if (threadIdx.x < (c.rows + kScaleRows - 1) / kScaleRows)
        a.pool.scales[to / kScaleRows + threadIdx.x] = a.pool.scales[from / kScaleRows + threadIdx.x];
}

// ---- rows as bf16 ------------------------------------------------------------------
constexpr int kReadThreads = 256;
constexpr int kReadUnroll = 4;   // eights of elements a thread has in flight

__device__ __forceinline__ uint4 widen8(uint2 codes, float scale) {
    const float4 a = e4m3_values(codes.x, scale), b = e4m3_values(codes.y, scale);
    return make_uint4(pack_bf16x2(a.x, a.y), pack_bf16x2(a.z, a.w), pack_bf16x2(b.x, b.y),
                      pack_bf16x2(b.z, b.w));
}

// A thread to kReadUnroll eights of a run's elements in the order of the output; the
// values of 8 bits are exact in bf16.  13,015 rows of 8 heads of 128 dimensions: 80 MB in
// 15.0 us, 13.2 behind the store that wrote them.
template <int D>
__global__ void __launch_bounds__(kReadThreads)
    sq_kv8_read_kernel(const __grid_constant__ Kv8ReadInlineArgs a, int parts) {
    grid_dependency_wait();
    grid_launch_dependents();
    const int part = blockIdx.x % parts, r = blockIdx.x / parts, kv = blockIdx.y;
    const RowRun run = a.runs ? a.runs[r] : a.inline_run[r];
    const Kv8Pool& p = a.pool;
    const int64_t page = run.row >> log2_of(p.P);
    const int slot = run.row & (p.P - 1);
    if (run.row < 0 || page >= p.num_pages || slot + run.n > p.P) {
        if (threadIdx.x == 0) set_error(a.err, kErrBounds);
        return;
    }
    constexpr int kEights = D / 8;
    const int64_t plane = plane_row(p, a.layer, page, kv, 0) + slot;
    uint4* out = reinterpret_cast<uint4*>((kv ? a.v : a.k) + (int64_t)run.first * p.Hkv * D);
    const int n = run.n * p.Hkv * kEights;
    uint4 x[kReadUnroll];
    float s[kReadUnroll];
#pragma unroll
    for (int u = 0; u < kReadUnroll; ++u) {
        const int i = (part * kReadUnroll + u) * kReadThreads + threadIdx.x;
        if (i >= n) continue;
        const int row = i / kEights, t = row / p.Hkv, head = row - t * p.Hkv;
        const int64_t at = plane + (int64_t)head * p.P + t;
        if (p.codes) {
            const uint2 c = *reinterpret_cast<const uint2*>(p.codes + at * D + i % kEights * 8);
            x[u] = make_uint4(c.x, c.y, 0, 0);
            s[u] = p.scales[at / kScaleRows];
        } else {
            x[u] = *reinterpret_cast<const uint4*>(a.wide + at * D + i % kEights * 8);
        }
    }
#pragma unroll
    for (int u = 0; u < kReadUnroll; ++u) {
        const int i = (part * kReadUnroll + u) * kReadThreads + threadIdx.x;
        if (i < n) out[i] = p.codes ? widen8(make_uint2(x[u].x, x[u].y), s[u]) : x[u];
    }
}

// Whole pages of one layer, a CTA to kReadThreads * kReadUnroll eights of a page.  60,513
// tokens, 8 heads of 128 dimensions: 372 MB in 55 us, at the copy rate.
template <int D>
__global__ void __launch_bounds__(kReadThreads)
    sq_kv8_widen_kernel(const __grid_constant__ Kv8WidenArgs a, int parts) {
    grid_dependency_wait();
    grid_launch_dependents();
    const int part = blockIdx.x % parts, i0 = blockIdx.x / parts;
    int64_t page = a.pages[i0];
    if (page < 0 || page >= a.pool.num_pages) {
        if (threadIdx.x == 0) set_error(a.err, kErrBounds);
        page = 0;
    }
    constexpr int kEights = D / 8;
    const int n = 2 * a.pool.Hkv * a.pool.P * kEights;
    const int64_t row0 = plane_row(a.pool, a.layer, page, 0, 0);
    uint4* out = reinterpret_cast<uint4*>(a.out) + (int64_t)i0 * n;
    uint2 x[kReadUnroll];
    float s[kReadUnroll];
#pragma unroll
    for (int u = 0; u < kReadUnroll; ++u) {
        const int i = (part * kReadUnroll + u) * kReadThreads + threadIdx.x;
        if (i >= n) continue;
        x[u] = *(reinterpret_cast<const uint2*>(a.pool.codes + row0 * D) + i);
        s[u] = a.pool.scales[(row0 + i / kEights) / kScaleRows];
    }
#pragma unroll
    for (int u = 0; u < kReadUnroll; ++u) {
        const int i = (part * kReadUnroll + u) * kReadThreads + threadIdx.x;
        if (i < n) out[i] = widen8(x[u], s[u]);
    }
}

// ---- eviction --------------------------------------------------------------------
// A CTA takes one plane's tiles of a chunk in order, a batch of them at a time: their
// rows (a tile: all that a page gets) are read into shared memory, then written block
// by block, with the scale of the rows that are together now.  The batch after it is
// read meanwhile, which in-place compaction allows: rows only move towards the front, so
// what a tile is made of lies in no page of the tiles before it.
//
// What bounds it: the planes' chains of batches (a dense eviction of one sequence has
// L x 2 x Hkv of them, 256 here), and in each the work on its codes.  32,768 tokens of
// 16 layers, 8 x 128, 44% evicted on pages of 64: 786 us with a tile at a time, 638 with
// batches of four, 610 with their records read ahead, 382 with rows taken from scale to
// scale by fp16 products of their codes (3.1 TB/s).
constexpr int kEvictThreads = 256, kEvictWarps = kEvictThreads / 32;
constexpr int kBatchBytes = 36 << 10, kBatchMost = 16;

__host__ __device__ inline int evict_tile_bytes(int P, int D) { return P * (D + 4); }   // rows, scales
__host__ __device__ inline int evict_batch(int P, int D) {
    const int n = kBatchBytes / evict_tile_bytes(P, D);
    return n < 1 ? 1 : n > kBatchMost ? kBatchMost : n;
}
// Two batches and their tiles' records.
__host__ __device__ inline int evict_smem(int P, int D) {
    return 2 * evict_batch(P, D) * (evict_tile_bytes(P, D) + (int)sizeof(EvictTile));
}

template <int D>
__global__ void __launch_bounds__(kEvictThreads)
    sq_kv8_evict_kernel(const __grid_constant__ Kv8EvictArgs a) {
    grid_dependency_wait();
    grid_launch_dependents();
    extern __shared__ uint4 evict_tiles_smem[];
    const Kv8Pool& p = a.pool;
    const int P = p.P, lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const int planes = a.L * 2 * p.Hkv;
    const int plane = blockIdx.x % planes, chunk = blockIdx.x / planes;
    const int head = plane % p.Hkv, kv = plane / p.Hkv % 2, layer = plane / (2 * p.Hkv);
    constexpr int kVecs = D / 16;
    const int n_batch = evict_batch(P, D), tile_bytes = evict_tile_bytes(P, D);
    uint8_t* base = reinterpret_cast<uint8_t*>(evict_tiles_smem);
    auto rows_of = [&](int b, int i) { return base + (b * n_batch + i) * tile_bytes; };
    auto scales_of = [&](int b, int i) { return reinterpret_cast<float*>(rows_of(b, i) + P * D); };
    // (dst_page -1: none; piece_begin -1: zeros)
    EvictTile* recs = reinterpret_cast<EvictTile*>(base + 2 * n_batch * tile_bytes);
    const int t0 = a.chunk[chunk], t1 = a.chunk[chunk + 1];
    // A batch's tiles, row r of a page where its slot is; a warp or more to a tile, whose
    // records (a piece to a lane, the first 32 of them) it has read a batch ahead.
    const int share = max(1, kEvictWarps / n_batch), part = warp % share;
    constexpr int kMine = kBatchMost / kEvictWarps;   // tiles of a warp at most
    struct Record {
        EvictTile tile;
        EvictPiece piece;
        int end;
    } ahead[kMine];
    auto look_up = [&](int t) {
#pragma unroll
        for (int m = 0; m < kMine; ++m) {
            const int i = warp / share + m * (kEvictWarps / share);
            Record& r = ahead[m];
            r.tile = {-1, 0, 0, 0};
            r.end = 0;
            if (i >= n_batch || t + i >= t1) continue;
            r.tile = a.tiles[t + i];
            r.end = t + i + 1 < a.n_tiles ? a.tiles[t + i + 1].piece_begin : a.n_pieces;
            if (r.tile.piece_begin + lane < r.end) r.piece = a.pieces[r.tile.piece_begin + lane];
        }
    };
    auto read = [&](int t, int b) {
#pragma unroll
        for (int m = 0; m < kMine; ++m) {
            const int i = warp / share + m * (kEvictWarps / share);
            if (i >= n_batch) continue;
            EvictTile tile = ahead[m].tile;
            if (tile.dst_page != -1 &&
                ((uint64_t)tile.dst_page >= (uint64_t)p.num_pages || tile.dst_slot + tile.n_rows > P)) {
                if (lane == 0) set_error(a.err, kErrBounds);
                tile.dst_page = -1;
            }
            const int end = tile.dst_page >= 0 ? ahead[m].end : tile.piece_begin;
            for (int k = tile.piece_begin; k < end; ++k) {
                const int from_lane = k - tile.piece_begin;
                EvictPiece pc;
                if (from_lane < 32) {
                    pc.src_page = __shfl_sync(0xffffffffu, ahead[m].piece.src_page, from_lane);
                    pc.src_slot = __shfl_sync(0xffffffffu, ahead[m].piece.src_slot, from_lane);
                    pc.n_rows = __shfl_sync(0xffffffffu, ahead[m].piece.n_rows, from_lane);
                    pc.dst_row = __shfl_sync(0xffffffffu, ahead[m].piece.dst_row, from_lane);
                } else {
                    pc = a.pieces[k];
                }
                const int to = tile.dst_slot + pc.dst_row;
                if ((uint64_t)pc.src_page >= (uint64_t)p.num_pages || pc.src_slot + pc.n_rows > P ||
                    to + pc.n_rows > P) {
                    if (lane == 0) set_error(a.err, kErrBounds);
                    continue;
                }
                const int64_t from = plane_row(p, layer, pc.src_page, kv, head) + pc.src_slot;
                const uint32_t dst = smem_addr(rows_of(b, i) + to * D);
                const uint8_t* src = p.codes + from * D;
                for (int v = part * 32 + lane; v < pc.n_rows * kVecs; v += share * 32)
                    asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(dst + 16 * v), "l"(src + 16 * v)
                                 : "memory");
                const uint32_t sdst = smem_addr(scales_of(b, i) + to);
                for (int v = part * 32 + lane; v < pc.n_rows; v += share * 32)
                    asm volatile("cp.async.ca.shared.global [%0], [%1], 4;" ::"r"(sdst + 4 * v),
                                 "l"(p.scales + (from + v) / kScaleRows)
                                 : "memory");
            }
            if (tile.dst_page >= 0 && tile.piece_begin == ahead[m].end) tile.piece_begin = -1;
            if (part == 0 && lane == 0) recs[b * n_batch + i] = tile;
        }
        asm volatile("cp.async.commit_group;" ::: "memory");
        look_up(t + n_batch);
    };
    look_up(t0);
    read(t0, 0);
    const int page_blocks = P / kScaleRows;
    constexpr int kRowLanes = D / 16;              // 16 codes a lane
    constexpr int kRows = 32 / kRowLanes;          // rows of a warp at once
    constexpr int kPass = kScaleRows / kRows;
    for (int t = t0, b = 0; t < t1; t += n_batch, b ^= 1) {
        read(t + n_batch, b ^ 1);
        asm volatile("cp.async.wait_group 1;" ::: "memory");
        __syncthreads();
        for (int x = warp; x < n_batch * page_blocks; x += kEvictWarps) {
            const int i = x / page_blocks, blk = x - i * page_blocks;
            const EvictTile tile = recs[b * n_batch + i];
            const int r0 = tile.dst_slot, r1 = r0 + tile.n_rows;
            if (tile.dst_page < 0 || blk * kScaleRows >= r1 || (blk + 1) * kScaleRows <= r0) continue;
            const int64_t page_row = plane_row(p, layer, tile.dst_page, kv, head);
            uint8_t* codes = p.codes + (page_row + blk * kScaleRows) * D;
            float* scale = p.scales + (page_row / kScaleRows + blk);
            if (tile.piece_begin < 0) {
                // a block that keeps rows keeps its scale
                for (int u = 0; u < kPass; ++u) {
                    const int row = blk * kScaleRows + u * kRows + lane / kRowLanes;
                    if (row >= r0 && row < r1)
                        *reinterpret_cast<uint4*>(codes + (row - blk * kScaleRows) * D + lane % kRowLanes * 16) =
                            make_uint4(0, 0, 0, 0);
                }
                if (lane == 0 && blk * kScaleRows >= r0) *scale = power_of_two(kLeastScale);
                continue;
            }
            // rows before the tile's first stay where they are
            uint4 c[kPass];
            float s[kPass];
            const float old = blk * kScaleRows < r0 ? *scale : 0.f;
#pragma unroll
            for (int u = 0; u < kPass; ++u) {
                const int i8 = u * kRows + lane / kRowLanes, row = blk * kScaleRows + i8;
                c[u] = make_uint4(0, 0, 0, 0);
                s[u] = old;
                if (row >= r1) continue;
                if (row < r0) {
                    c[u] = *reinterpret_cast<const uint4*>(codes + i8 * D + lane % kRowLanes * 16);
                } else {
                    c[u] = *reinterpret_cast<const uint4*>(rows_of(b, i) + row * D + lane % kRowLanes * 16);
                    s[u] = scales_of(b, i)[row];
                }
            }
            float size = 0.f;
#pragma unroll
            for (int u = 0; u < kPass; ++u) size = fmaxf(size, code_size(c[u]) * s[u]);
            size = warp_size(size);
            const int e = scale_exponent(size);
            const float now = power_of_two(e);
#pragma unroll
            for (int u = 0; u < kPass; ++u) {
                const int i8 = u * kRows + lane / kRowLanes, row = blk * kScaleRows + i8;
                if (row >= r1 || (row < r0 && now == old)) continue;
                if (s[u] != now) c[u] = rescaled(c[u], s[u], e);
                *reinterpret_cast<uint4*>(codes + i8 * D + lane % kRowLanes * 16) = c[u];
            }
            if (lane == 0) *scale = now;
        }
        __syncthreads();
    }
}

template <typename... P, typename... A>
cudaError_t launch_after(void (*kernel)(P...), dim3 grid, unsigned block, int smem, cudaStream_t st,
                         const A&... args) {
    cudaLaunchAttribute at;
    at.id = cudaLaunchAttributeProgrammaticStreamSerialization;
    at.val.programmaticStreamSerializationAllowed = 1;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = grid;
    cfg.blockDim = dim3(block);
    cfg.dynamicSmemBytes = smem;
    cfg.stream = st;
    cfg.attrs = &at;
    cfg.numAttrs = 1;
    return cudaLaunchKernelEx(&cfg, kernel, args...);
}

template <int D>
cudaError_t store(const Kv8StoreInlineArgs& a, cudaStream_t st) {
    const int64_t warps = (int64_t)a.n_runs * a.blocks * StoreTasks<D>(a.Hq, a.Hkv, a.most).total;
    constexpr int per = kStoreThreads / 32;
    const dim3 grid((unsigned)((warps + per - 1) / per), (unsigned)a.n_layers);
    return launch_after(a.interleaved ? sq_kv8_store_kernel<D, true> : sq_kv8_store_kernel<D, false>, grid,
                        kStoreThreads, 0, st, a);
}

}  // namespace

cudaError_t kv8_prepare(int D) {
    int most = 0;
    for (int P = 8; P <= 256; P *= 2) most = std::max(most, evict_smem(P, D));
    return cudaFuncSetAttribute(D == 128 ? sq_kv8_evict_kernel<128> : sq_kv8_evict_kernel<64>,
                                cudaFuncAttributeMaxDynamicSharedMemorySize, most);
}

cudaError_t launch_kv8_store(const Kv8StoreInlineArgs& a, int D, cudaStream_t st) {
    if (a.n_runs == 0) return cudaSuccess;
    return D == 128 ? store<128>(a, st) : store<64>(a, st);
}

cudaError_t launch_kv8_copy(const Kv8CopyArgs& a, int D, cudaStream_t st) {
    const unsigned grid = std::max(1u, (unsigned)a.n_cow * a.L * 2 * a.pool.Hkv);
    return launch_after(sq_kv8_copy_kernel, dim3(grid), kCopyThreads, 0, st, a, D);
}

cudaError_t launch_kv8_read(const Kv8ReadInlineArgs& a, int D, cudaStream_t st) {
    if (a.n_runs == 0) return cudaSuccess;
    const int eights = a.most * a.pool.Hkv * (D / 8), per = kReadThreads * kReadUnroll;
    const int parts = (eights + per - 1) / per;
    const dim3 grid((unsigned)a.n_runs * parts, 2);
    return launch_after(D == 128 ? sq_kv8_read_kernel<128> : sq_kv8_read_kernel<64>, grid, kReadThreads, 0, st, a,
                        parts);
}

cudaError_t launch_kv8_widen(const Kv8WidenArgs& a, int D, cudaStream_t st) {
    if (a.n == 0) return cudaSuccess;
    const int eights = 2 * a.pool.Hkv * a.pool.P * (D / 8), per = kReadThreads * kReadUnroll;
    const int parts = (eights + per - 1) / per;
    return launch_after(D == 128 ? sq_kv8_widen_kernel<128> : sq_kv8_widen_kernel<64>, dim3((unsigned)a.n * parts),
                        kReadThreads, 0, st, a, parts);
}

cudaError_t launch_kv8_evict(const Kv8EvictArgs& a, int D, cudaStream_t st) {
    const dim3 grid((unsigned)a.n_chunks * a.L * 2 * a.pool.Hkv);
    return launch_after(D == 128 ? sq_kv8_evict_kernel<128> : sq_kv8_evict_kernel<64>, grid, kEvictThreads,
                        evict_smem(a.pool.P, D), st, a);
}

}  // namespace sq
