// fake_operators.cpp with stand-ins for the launchers of 8-bit rows: a code is the low
// byte of the element that it is given, a block's scale the rows that the block held
// when it was written; moves, copies and reads take both along.
#define cudaEventQuery event_query
#define cudaStreamIsCapturing stream_capturing
#include "fake_operators.cpp"
#undef cudaEventQuery
#undef cudaStreamIsCapturing

#include <algorithm>

#include "../paper_2602_22603_gb300/csrc/kernels/kv8.hpp"

namespace sq {

enum { kStore8, kCopy8, kRead8, kWiden8, kEvict8 };
static int g_fail8 = -1;
static int64_t g_bad = 0;   // runs that a launch should not be given
static bool fails8(int kind) {
    if (g_fail8 != kind) return false;
    g_fail8 = -1;
    return true;
}
// Uses of the pool's pages, as of other memory (see fake_device.cpp).
static std::map<int, std::vector<Use>> g_pages;
static int64_t g_page_races = 0;
static void use_page(cudaStream_t st, const Clock& c, int page, bool write) {
    for (const Use& u : g_pages[page]) {
        auto known = c.find(u.stream);
        if ((u.write || write) && (known == c.end() || known->second < u.seq)) ++g_page_races;
    }
    g_pages[page].push_back({st, c.at(st), write});
}
static std::vector<int> g_early;   // pages that the last launch of single tokens was to leave to its wait
static int g_early_on = 0;
static int64_t plane8(const Kv8Pool& p, int layer, int page, int kv, int head) {
    return (((layer * p.num_pages + page) * 2 + kv) * p.Hkv + head) * (int64_t)p.P;
}

cudaError_t kv8_prepare(int) { return cudaSuccess; }
cudaError_t launch_kv8_store(const Kv8StoreInlineArgs& a, int D, cudaStream_t st) {
    if (fails8(kStore8)) return cudaErrorLaunchFailure;
    const Clock& c = tick(st);
    if (a.runs) use(st, c, a.runs, false);
    for (int r = 0; r < a.n_runs; ++r) {
        const RowRun all = a.runs ? a.runs[r] : a.inline_run[r];
        const int page = all.row / a.pool.P;
        if (all.n < 1 || all.n > kRunRows || page < 0 || page >= a.pool.num_pages ||
            all.row / std::min(a.pool.P, kRunRows) != (all.row + all.n - 1) / std::min(a.pool.P, kRunRows))
            ++g_bad;
        use_page(st, c, page, true);
        for (int b = 0; b < a.blocks; ++b) {
            const int b0 = all.row / kScaleRows * kScaleRows + b * kScaleRows;
            const int from = std::max(all.row, b0), end = std::min(all.row + all.n, b0 + kScaleRows);
            if (end - from > a.most) ++g_bad;
            if (b + 1 == a.blocks && end < all.row + all.n) ++g_bad;
            if (end <= from) continue;
            const int first = all.first + from - all.row, slot = from % a.pool.P;
            for (int l = 0; l < a.n_layers; ++l)
                for (int kv = 0; kv < 2; ++kv)
                    for (int h = 0; h < a.Hkv; ++h) {
                        const int64_t row = plane8(a.pool, a.layer + l, page, kv, h) + slot;
                        const __nv_bfloat16* src = (kv ? a.v : a.k) + l * a.layer_stride;
                        for (int i = 0; i < end - from; ++i)
                            for (int e = 0; e < D; ++e)
                                a.pool.codes[(row + i) * D + e] = *reinterpret_cast<const uint8_t*>(
                                    src + (first + i) * (kv ? a.v_stride : a.k_stride) + h * D + e);
                        a.pool.scales[row / kScaleRows] = (float)(slot % kScaleRows + end - from);
                    }
        }
    }
    return cudaSuccess;
}
cudaError_t launch_kv8_copy(const Kv8CopyArgs& a, int D, cudaStream_t st) {
    if (fails8(kCopy8)) return cudaErrorLaunchFailure;
    const Clock& c = tick(st);
    for (int i = 0; i < a.lens.n; ++i) *a.lens.ptr[i] = a.lens.val[i];
    for (int i = 0; i < a.n_cow; ++i) {
        use_page(st, c, a.cow[i].src_page, false);
        use_page(st, c, a.cow[i].dst_page, true);
    }
    for (int i = 0; i < a.n_cow; ++i)
        for (int l = 0; l < a.L; ++l)
            for (int x = 0; x < 2 * a.pool.Hkv; ++x) {
                const int64_t from = plane8(a.pool, l, a.cow[i].src_page, x / a.pool.Hkv, x % a.pool.Hkv);
                const int64_t to = plane8(a.pool, l, a.cow[i].dst_page, x / a.pool.Hkv, x % a.pool.Hkv);
                std::memcpy(a.pool.codes + to * D, a.pool.codes + from * D, (size_t)a.cow[i].rows * D);
                for (int b = 0; b * kScaleRows < a.cow[i].rows; ++b)
                    a.pool.scales[to / kScaleRows + b] = a.pool.scales[from / kScaleRows + b];
            }
    return cudaSuccess;
}
cudaError_t launch_kv8_read(const Kv8ReadInlineArgs& a, int D, cudaStream_t st) {
    if (fails8(kRead8)) return cudaErrorLaunchFailure;
    const Clock& c = tick(st);
    if (a.runs) use(st, c, a.runs, false);
    for (int r = 0; r < a.n_runs; ++r) {
        const RowRun run = a.runs ? a.runs[r] : a.inline_run[r];
        if (run.n < 1 || run.n > a.most || run.row % a.pool.P + run.n > a.pool.P) ++g_bad;
        for (int kv = 0; kv < 2; ++kv)
            for (int i = 0; i < run.n; ++i)
                for (int h = 0; h < a.pool.Hkv; ++h) {
                    const int64_t row = plane8(a.pool, a.layer, run.row / a.pool.P, kv, h) + run.row % a.pool.P + i;
                    uint16_t* out = reinterpret_cast<uint16_t*>(kv ? a.v : a.k) +
                                    ((int64_t)(run.first + i) * a.pool.Hkv + h) * D;
                    for (int e = 0; e < D; ++e)
                        out[e] = a.pool.codes ? a.pool.codes[row * D + e]
                                              : reinterpret_cast<const uint16_t*>(a.wide)[row * D + e];
                }
    }
    return cudaSuccess;
}
static int g_wide = 0;   // pages of the last widening
cudaError_t launch_kv8_widen(const Kv8WidenArgs& a, int, cudaStream_t st) {
    if (fails8(kWiden8)) return cudaErrorLaunchFailure;
    const Clock& c = tick(st);
    use(st, c, a.pages, false);
    use(st, c, a.out, true);
    g_wide = a.n;
    for (int i = 0; i < a.n; ++i)
        if (a.pages[i] < 0 || a.pages[i] >= a.pool.num_pages) ++g_bad;
    return cudaSuccess;
}
cudaError_t blocks_kv8_prepare(int) { return cudaSuccess; }
cudaError_t launch_blocks_kv8(const CUtensorMap& m, const CUtensorMap& q, const BlockShortKv8Args& a, int D,
                              cudaStream_t st) {
    if (!a.scales) ++g_bad;
    g_wide = 0;
    return launch_blocks(m, q, a, D, true, st);
}
cudaError_t launch_kv8_evict(const Kv8EvictArgs& a, int D, cudaStream_t st) {
    if (fails8(kEvict8)) return cudaErrorLaunchFailure;
    const Clock& c = tick(st);
    use(st, c, a.tiles, false);
    const Kv8Pool& p = a.pool;
    for (int l = 0; l < a.L; ++l)
        for (int x = 0; x < 2 * p.Hkv; ++x)
            for (int t = 0; t < a.n_tiles; ++t) {
                const EvictTile tile = a.tiles[t];
                if (l + x == 0) use_page(st, c, tile.dst_page, true);
                const int end = t + 1 < a.n_tiles ? a.tiles[t + 1].piece_begin : a.n_pieces;
                std::vector<uint8_t> rows((size_t)tile.n_rows * D, 0);
                for (int k = tile.piece_begin; k < end; ++k)
                    std::memcpy(rows.data() + a.pieces[k].dst_row * D,
                                p.codes + (plane8(p, l, a.pieces[k].src_page, x / p.Hkv, x % p.Hkv) +
                                           a.pieces[k].src_slot) * D,
                                (size_t)a.pieces[k].n_rows * D);
                const int64_t to = plane8(p, l, tile.dst_page, x / p.Hkv, x % p.Hkv) + tile.dst_slot;
                std::memcpy(p.codes + to * D, rows.data(), rows.size());
            }
    return cudaSuccess;
}
static int g_rows = 0;   // rows of its longest segment
cudaError_t launch_decode_kv8(const CUtensorMap& m, const DecodeKv8Args& a, int n, int D, cudaStream_t st) {
    if (!a.scales) ++g_bad;
    const cudaError_t e = launch_decode(m, a, n, D, st);
    if (e != cudaSuccess) return e;
    g_early.assign(a.unsafe, a.unsafe + (a.kv_early ? a.n_unsafe : 0));
    g_early_on = a.kv_early;
    g_rows = 0;
    for (int i = 0; i < a.cta_begin[n]; ++i) {
        const DecodeSeg& s = a.segs[a.items[i].seg];
        g_rows = std::max(g_rows, (int)s.n_tok);
        for (int p = 0; p < s.n_pages; ++p) use_page(st, g_streams[st], a.page_ids[s.page_off + p], false);
    }
    return e;
}

}  // namespace sq

EXPORT void fake_fail8(int kind) { sq::g_fail8 = kind; }
EXPORT int64_t fake_bad() { return sq::g_bad; }
EXPORT int fake_wide() { return sq::g_wide; }
EXPORT int64_t fake_page_races() { return sq::g_page_races; }
EXPORT void fake_new_pages() { sq::g_pages.clear(), sq::g_page_races = 0; }
// Whether the last launch of single tokens was to load a page before its wait.
EXPORT int fake_early(int page) {
    return sq::g_early_on && std::find(sq::g_early.begin(), sq::g_early.end(), page) == sq::g_early.end();
}
EXPORT int fake_rows() { return sq::g_rows; }
static bool g_done = false, g_graph = false;
EXPORT void fake_done(int done) { g_done = done; }       // what events answer
EXPORT void fake_graph(int graph) { g_graph = graph; }   // streams are captured
extern "C" cudaError_t cudaEventQuery(cudaEvent_t) { return g_done ? cudaSuccess : cudaErrorNotReady; }
extern "C" cudaError_t cudaStreamIsCapturing(cudaStream_t, cudaStreamCaptureStatus* s) {
    return *s = g_graph ? cudaStreamCaptureStatusActive : cudaStreamCaptureStatusNone, cudaSuccess;
}
