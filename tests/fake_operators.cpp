// fake_device.cpp with stand-ins for the launchers of the calls around a model's
// attention: they note the buffers they use, and stores write their rows' keys
// and values as they are (no norm, no rotation).
#include "fake_device.cpp"

#include "../paper_2602_22603_gb300/csrc/kernels/operators.hpp"

namespace sq {

enum { kNorm = 6, kBlocks = 7 };

cudaError_t blocks_prepare(int) { return cudaSuccess; }

static void store(const NormRopeArgs& a, const RowPlace* places, int D) {
    for (int t = 0; t < a.n; ++t)
        for (int h = 0; h < a.Hkv; ++h) {
            const int page = places[t].row / a.P, slot = places[t].row % a.P;
            std::memcpy(a.pool + row_at(a.num_pages, a.Hkv, a.P, D, a.layer, page, 0, h, slot),
                        a.k + t * a.k_stride + h * D, (size_t)D * 2);
            std::memcpy(a.pool + row_at(a.num_pages, a.Hkv, a.P, D, a.layer, page, 1, h, slot),
                        a.v + t * a.v_stride + h * D, (size_t)D * 2);
        }
}

cudaError_t launch_norm_rope(const NormRopeArgs& a, int D, bool to_pool, cudaStream_t st) {
    if (fails(kNorm)) return cudaErrorLaunchFailure;
    const Clock& c = tick(st);
    if (!to_pool) return cudaSuccess;
    use(st, c, a.places, false);
    store(a, a.places, D);
    return cudaSuccess;
}
cudaError_t launch_norm_rope_inline(const NormRopeInlineArgs& a, int D, cudaStream_t st) {
    if (fails(kNorm)) return cudaErrorLaunchFailure;
    tick(st);
    store(a, a.inline_place, D);
    return cudaSuccess;
}
int norm_rope_grad_ctas(int32_t n, int32_t, int32_t, int, int num_sms) { return n < num_sms ? n + 1 : num_sms; }
cudaError_t launch_norm_rope_grad(const NormRopeGradArgs& a, int, cudaStream_t st) {
    if (fails(kNorm)) return cudaErrorLaunchFailure;
    const Clock& c = tick(st);
    use(st, c, a.part, true);
    return cudaSuccess;
}

// What the last query-block launch was allowed to read early (-1: nothing).
static int g_unsafe = -1;
cudaError_t launch_blocks(const CUtensorMap&, const CUtensorMap&, const BlockShortArgs& a, int, bool,
                          cudaStream_t st) {
    if (fails(kBlocks)) return cudaErrorLaunchFailure;
    const Clock& c = tick(st);
    use(st, c, a.tiles, false);
    const BlockItem* items = reinterpret_cast<const BlockItem*>(a.items);
    bool split = false;
    for (int i = 0; i < a.n_items; ++i) split |= items[i].part >= 0;
    if (split) use(st, c, a.part_o, true);
    g_unsafe = a.kv_early ? a.n_unsafe : -1;
    return cudaSuccess;
}
cudaError_t launch_blocks_combine(const BlockCombineArgs& a, int, cudaStream_t st) {
    if (fails(kCombine)) return cudaErrorLaunchFailure;
    const Clock& c = tick(st);
    use(st, c, a.merges, false);
    use(st, c, a.part_o, false);
    return cudaSuccess;
}

}  // namespace sq

EXPORT int fake_unsafe() { return sq::g_unsafe; }
