// Launches of masked prefill attention: the queries of one sequence
// (prefill_kernel.cuh has the kernels).
#include "prefill_kernel.cuh"

namespace sq {

template <int D>
static cudaError_t prepare() {
    cudaError_t e = cudaFuncSetAttribute(dev::sq_prefill_kernel<D, PrefillArgs>,
                                         cudaFuncAttributeMaxDynamicSharedMemorySize,
                                         dev::PreCfg<D, 0>::kSmemBytes);
    if (e != cudaSuccess) return e;
    e = cudaFuncSetAttribute(dev::sq_prefill_kernel<D, PrefillShortArgs>, cudaFuncAttributeMaxDynamicSharedMemorySize,
                             dev::PreCfg<D, dev::kOneTile>::kSmemBytes);
    if (e != cudaSuccess) return e;
    e = cudaFuncSetAttribute(dev::sq_prefill_kernel<D, PrefillHideArgs>, cudaFuncAttributeMaxDynamicSharedMemorySize,
                             dev::PreCfg<D, dev::kHides>::kSmemBytes);
    if (e != cudaSuccess) return e;
    e = cudaFuncSetAttribute(dev::sq_prefill_kernel<D, PrefillHideShortArgs>,
                             cudaFuncAttributeMaxDynamicSharedMemorySize,
                             dev::PreCfg<D, dev::kHides | dev::kOneTile>::kSmemBytes);
    if (e != cudaSuccess) return e;
    // the same split of L1 and shared memory as the prefill kernel's: they take
    // turns on every SM
    e = cudaFuncSetAttribute(dev::sq_prefill_combine_kernel<D, 2, 24, PrefillCombineArgs>,
                             cudaFuncAttributePreferredSharedMemoryCarveout,
                             cudaSharedmemCarveoutMaxShared);
    if (e != cudaSuccess) return e;
    return cudaFuncSetAttribute(dev::sq_prefill_combine_kernel<D, D / 32, dev::kCombineFew, PrefillCombineArgs>,
                                cudaFuncAttributePreferredSharedMemoryCarveout,
                                cudaSharedmemCarveoutMaxShared);
}

int prefill_smem_bytes(int D) {
    return D == 128 ? dev::PreCfg<128, 0>::kSmemBytes : dev::PreCfg<64, 0>::kSmemBytes;
}

cudaError_t prefill_prepare(int D) { return D == 128 ? prepare<128>() : prepare<64>(); }

cudaError_t launch_prefill(const CUtensorMap& pool_map, const CUtensorMap& qmap,
                           const PrefillShortArgs& a, int D, cudaStream_t st) {
    const unsigned grid = (unsigned)a.n_items;
    if (grid == 0) return cudaSuccess;
    // a programmatic dependent of whatever precedes it: its barrier and tensor
    // memory set-up overlaps that work's tail.  Before its wait it reads only a
    // plan that was on the device already (plan_ready), and, in the short
    // instance, keys and values that no running work writes (kv_early).
    cudaLaunchAttribute at;
    at.id = cudaLaunchAttributeProgrammaticStreamSerialization;
    at.val.programmaticStreamSerializationAllowed = 1;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3(grid);
    cfg.stream = st;
    cfg.attrs = &at;
    cfg.numAttrs = 1;
    auto launch = [&](auto cfg_of, auto kernel, const auto& args) {
        using C = decltype(cfg_of);
        cfg.blockDim = dim3(C::kThreads);
        cfg.dynamicSmemBytes = C::kSmemBytes;
        return cudaLaunchKernelEx(&cfg, kernel, pool_map, qmap, args);
    };
    const PrefillArgs& base = a;
    const bool one = a.n_q <= a.BP;  // every query in tile a of the only CTA tile
    if (a.hides) {
        PrefillHideShortArgs s;
        static_cast<PrefillShortArgs&>(s) = a;
        PrefillHideArgs b;
        static_cast<PrefillArgs&>(b) = a;
        constexpr int kH = dev::kHides, kHO = dev::kHides | dev::kOneTile;
        if (D == 128)
            return one ? launch(dev::PreCfg<128, kHO>{}, dev::sq_prefill_kernel<128, PrefillHideShortArgs>, s)
                       : launch(dev::PreCfg<128, kH>{}, dev::sq_prefill_kernel<128, PrefillHideArgs>, b);
        return one ? launch(dev::PreCfg<64, kHO>{}, dev::sq_prefill_kernel<64, PrefillHideShortArgs>, s)
                   : launch(dev::PreCfg<64, kH>{}, dev::sq_prefill_kernel<64, PrefillHideArgs>, b);
    }
    if (D == 128)
        return one ? launch(dev::PreCfg<128, dev::kOneTile>{}, dev::sq_prefill_kernel<128, PrefillShortArgs>, a)
                   : launch(dev::PreCfg<128, 0>{}, dev::sq_prefill_kernel<128, PrefillArgs>, base);
    return one ? launch(dev::PreCfg<64, dev::kOneTile>{}, dev::sq_prefill_kernel<64, PrefillShortArgs>, a)
               : launch(dev::PreCfg<64, 0>{}, dev::sq_prefill_kernel<64, PrefillArgs>, base);
}

cudaError_t launch_prefill_combine(const PrefillCombineArgs& a, int D, cudaStream_t st) {
    const bool few = a.max_splits <= dev::kCombineFew;
    const int64_t warps = (int64_t)a.n_merges * a.rows * (few ? 1 : D / 64);
    const int per = dev::kCombineThreads / 32;
    const unsigned grid = (unsigned)((warps + per - 1) / per);
    if (grid == 0) return cudaSuccess;
    // scheduled while the prefill kernel's last CTAs run; waits for them
    cudaLaunchAttribute at;
    at.id = cudaLaunchAttributeProgrammaticStreamSerialization;
    at.val.programmaticStreamSerializationAllowed = 1;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3(grid);
    cfg.blockDim = dim3(dev::kCombineThreads);
    cfg.stream = st;
    cfg.attrs = &at;
    cfg.numAttrs = 1;
    constexpr int kF = dev::kCombineFew;
    if (D == 128)
        return few ? cudaLaunchKernelEx(&cfg, dev::sq_prefill_combine_kernel<128, 4, kF, PrefillCombineArgs>, a)
                   : cudaLaunchKernelEx(&cfg, dev::sq_prefill_combine_kernel<128, 2, 24, PrefillCombineArgs>, a);
    return few ? cudaLaunchKernelEx(&cfg, dev::sq_prefill_combine_kernel<64, 2, kF, PrefillCombineArgs>, a)
               : cudaLaunchKernelEx(&cfg, dev::sq_prefill_combine_kernel<64, 2, 24, PrefillCombineArgs>, a);
}

}  // namespace sq
