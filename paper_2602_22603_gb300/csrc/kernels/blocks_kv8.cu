// Launches of attention for query blocks of one tile over rows in 8 bits
// (prefill_kernel.cuh; see blocks.cu for bf16 rows).
#include "kv8.hpp"
#include "prefill_kernel.cuh"

namespace sq {
namespace {

// The register split of the kernel's roles draws on what the block is launched with, so
// that is checked here.
template <int D, typename Args>
cudaError_t prepare_one() {
    auto kernel = dev::sq_prefill_kernel<D, Args>;
    using C = dev::PreCfg<D, dev::ModeOf<Args>::value>;
    cudaFuncAttributes at;
    cudaError_t e = cudaFuncGetAttributes(&at, kernel);
    if (e != cudaSuccess) return e;
    if (at.numRegs * C::kThreads < C::kAllRegs) return cudaErrorInvalidConfiguration;
    return cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, C::kSmemBytes);
}

template <int D>
cudaError_t prepare() {
    const cudaError_t e = D == 128 ? prepare_one<128, BlockShortKv8Args>() : cudaSuccess;
    return e == cudaSuccess ? prepare_one<D, BlockShortKv8Args2>() : e;
}

// A programmatic dependent of whatever precedes it.
template <int D, typename Args>
cudaError_t launch_one(const CUtensorMap& pool_map, const CUtensorMap& qmap, const Args& a, cudaStream_t st) {
    using C = dev::PreCfg<D, dev::ModeOf<Args>::value>;
    cudaLaunchAttribute at;
    at.id = cudaLaunchAttributeProgrammaticStreamSerialization;
    at.val.programmaticStreamSerializationAllowed = 1;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)a.n_ctas);
    cfg.blockDim = dim3(C::kThreads);
    cfg.dynamicSmemBytes = C::kSmemBytes;
    cfg.stream = st;
    cfg.attrs = &at;
    cfg.numAttrs = 1;
    return cudaLaunchKernelEx(&cfg, dev::sq_prefill_kernel<D, Args>, pool_map, qmap, a);
}

template <int D>
cudaError_t launch_d(const CUtensorMap& pool_map, const CUtensorMap& qmap, const BlockShortKv8Args& a,
                     cudaStream_t st) {
    // (two producer warps as for bf16 rows)
    if constexpr (D == 128)
        if (a.n_pieces <= 2) return launch_one<D>(pool_map, qmap, a, st);
    BlockShortKv8Args2 s;
    static_cast<BlockShortKv8Args&>(s) = a;
    return launch_one<D>(pool_map, qmap, s, st);
}

}  // namespace

cudaError_t blocks_kv8_prepare(int D) { return D == 128 ? prepare<128>() : prepare<64>(); }

cudaError_t launch_blocks_kv8(const CUtensorMap& pool_map, const CUtensorMap& qmap, const BlockShortKv8Args& a,
                              int D, cudaStream_t st) {
    if (a.n_items == 0) return cudaSuccess;
    return D == 128 ? launch_d<128>(pool_map, qmap, a, st) : launch_d<64>(pool_map, qmap, a, st);
}

}  // namespace sq
