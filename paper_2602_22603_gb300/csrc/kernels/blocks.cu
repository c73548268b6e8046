// Launches of attention for query blocks: the newest tokens of a batch of
// sequences with sliding windows, sinks and drafted trees, by the prefill kernel's
// block instances (prefill_kernel.cuh).
#include "prefill_kernel.cuh"

namespace sq {
namespace {

template <int D, typename Args>
cudaError_t prepare_one() {
    return cudaFuncSetAttribute(dev::sq_prefill_kernel<D, Args>, cudaFuncAttributeMaxDynamicSharedMemorySize,
                                dev::PreCfg<D, dev::ModeOf<Args>::value>::kSmemBytes);
}

template <int D>
cudaError_t prepare() {
    cudaError_t e = prepare_one<D, BlockArgs>();
    if (e == cudaSuccess && D == 128) e = prepare_one<128, BlockShortArgs>();
    if (e == cudaSuccess) e = prepare_one<D, BlockArgs2>();
    if (e == cudaSuccess) e = prepare_one<D, BlockShortArgs2>();
    // (the merging kernels share every SM with the kernel above)
    if (e == cudaSuccess)
        e = cudaFuncSetAttribute(dev::sq_prefill_combine_kernel<D, 2, 24, BlockCombineArgs>,
                                 cudaFuncAttributePreferredSharedMemoryCarveout, cudaSharedmemCarveoutMaxShared);
    if (e == cudaSuccess)
        e = cudaFuncSetAttribute(dev::sq_prefill_combine_kernel<D, D / 32, dev::kCombineFew, BlockCombineArgs>,
                                 cudaFuncAttributePreferredSharedMemoryCarveout, cudaSharedmemCarveoutMaxShared);
    return e;
}

// A programmatic dependent of whatever precedes it (its set-up overlaps that
// work's tail).
template <typename... P, typename... A>
cudaError_t launch_after(void (*kernel)(P...), unsigned grid, unsigned block, int smem, cudaStream_t st,
                         const A&... args) {
    cudaLaunchAttribute at;
    at.id = cudaLaunchAttributeProgrammaticStreamSerialization;
    at.val.programmaticStreamSerializationAllowed = 1;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3(grid);
    cfg.blockDim = dim3(block);
    cfg.dynamicSmemBytes = smem;
    cfg.stream = st;
    cfg.attrs = &at;
    cfg.numAttrs = 1;
    return cudaLaunchKernelEx(&cfg, kernel, args...);
}

template <int D, typename Args>
cudaError_t launch_one(const CUtensorMap& pool_map, const CUtensorMap& qmap, const Args& a, cudaStream_t st) {
    using C = dev::PreCfg<D, dev::ModeOf<Args>::value>;
    return launch_after(dev::sq_prefill_kernel<D, Args>, (unsigned)a.n_ctas, C::kThreads, C::kSmemBytes, st,
                        pool_map, qmap, a);
}

}  // namespace

cudaError_t blocks_prepare(int D) { return D == 128 ? prepare<128>() : prepare<64>(); }

template <int D>
static cudaError_t launch_d(const CUtensorMap& pool_map, const CUtensorMap& qmap, const BlockShortArgs& a,
                            bool one, cudaStream_t st) {
    // (two producer warps: see block_produce)
    if (one && (D == 64 || a.n_pieces > 2)) {
        BlockShortArgs2 s;
        static_cast<BlockShortArgs&>(s) = a;
        return launch_one<D>(pool_map, qmap, s, st);
    }
    if constexpr (D == 128)
        if (one) return launch_one<D>(pool_map, qmap, a, st);
    if (a.n_pieces > 2) {
        BlockArgs2 s;
        static_cast<BlockArgs&>(s) = a;
        return launch_one<D>(pool_map, qmap, s, st);
    }
    const BlockArgs& base = a;
    return launch_one<D>(pool_map, qmap, base, st);
}

// one: every item's queries fit in one query tile
cudaError_t launch_blocks(const CUtensorMap& pool_map, const CUtensorMap& qmap, const BlockShortArgs& a,
                          int D, bool one, cudaStream_t st) {
    if (a.n_items == 0) return cudaSuccess;
    return D == 128 ? launch_d<128>(pool_map, qmap, a, one, st) : launch_d<64>(pool_map, qmap, a, one, st);
}

cudaError_t launch_blocks_combine(const BlockCombineArgs& a, int D, cudaStream_t st) {
    const bool few = a.max_splits <= dev::kCombineFew;
    const int64_t warps = (int64_t)a.n_merges * a.rows * (few ? 1 : D / 64);
    const int per = dev::kCombineThreads / 32;
    const unsigned grid = (unsigned)((warps + per - 1) / per);
    if (grid == 0) return cudaSuccess;
    constexpr int kF = dev::kCombineFew;
    auto run = [&](auto kernel) { return launch_after(kernel, grid, dev::kCombineThreads, 0, st, a); };
    if (D == 128)
        return few ? run(dev::sq_prefill_combine_kernel<128, 4, kF, BlockCombineArgs>)
                   : run(dev::sq_prefill_combine_kernel<128, 2, 24, BlockCombineArgs>);
    return few ? run(dev::sq_prefill_combine_kernel<64, 2, kF, BlockCombineArgs>)
               : run(dev::sq_prefill_combine_kernel<64, 2, 24, BlockCombineArgs>);
}

}  // namespace sq
