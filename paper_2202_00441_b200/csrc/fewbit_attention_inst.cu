// The attention kernels for one 16-bit type (FEWBIT_ATTN_F16: binary16, else bfloat16), with plain scores or with caps, biases
// and masks (FEWBIT_ATTN_SCORES).
#include <atomic>

#include "fewbit_attention.cuh"
#include "fewbit_attention_launch.h"

namespace fewbit {
bool pdl_enabled();

namespace attn {
namespace {

#if FEWBIT_ATTN_F16
using T = __half;
#else
using T = __nv_bfloat16;
#endif

template <auto kernel, int smem>
cudaError_t launch(const Params &p, unsigned grid, unsigned cluster, cudaStream_t st) {
    static std::atomic<unsigned long long> ready{0};                  // devices (up to 64) whose limit has been raised
    int dev = 0;
    cudaError_t err = cudaGetDevice(&dev);
    if (err != cudaSuccess) return err;
    const unsigned long long bit = dev < 64 ? 1ull << dev : 0;
    if ((ready.load(std::memory_order_relaxed) & bit) == 0) {
        err = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, smem);
        if (err != cudaSuccess) return err;
        ready.fetch_or(bit, std::memory_order_relaxed);
    }
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3(grid);
    cfg.blockDim = dim3(kThreadsAttn);
    cfg.dynamicSmemBytes = smem;
    cfg.stream = st;
    cudaLaunchAttribute attr[2];
    cfg.attrs = attr;
    if (pdl_enabled()) {
        attr[cfg.numAttrs].id = cudaLaunchAttributeProgrammaticStreamSerialization;
        attr[cfg.numAttrs++].val.programmaticStreamSerializationAllowed = 1;
    }
    if (cluster > 1) {
        attr[cfg.numAttrs].id = cudaLaunchAttributeClusterDimension;
        attr[cfg.numAttrs].val.clusterDim.x = cluster;
        attr[cfg.numAttrs].val.clusterDim.y = attr[cfg.numAttrs].val.clusterDim.z = 1;
        ++cfg.numAttrs;
    }
    return cudaLaunchKernelEx(&cfg, kernel, p);
}

template <int DIM, int MODE>
cudaError_t launch_one(Kernel which, const Params &p, unsigned grid, cudaStream_t st) {
    switch (which) {
    case Kernel::forward: return launch<attention_fwd_kernel<T, DIM, MODE>, fwd_smem<DIM>()>(p, grid * p.split, p.split, st);
    case Kernel::dq: return launch<attention_dq_kernel<T, DIM, MODE>, dq_smem<DIM>()>(p, grid * p.split, p.split, st);
    default:
        if constexpr (MODE == 2) {
            if (which == Kernel::dkv_bias) return launch<attention_dkv_kernel<T, DIM, 3>, dkv_smem<DIM>()>(p, grid * p.split, p.split, st);
        }
        return launch<attention_dkv_kernel<T, DIM, MODE>, dkv_smem<DIM>()>(p, grid * p.split, p.split, st);
    }
}

}  // namespace

#if FEWBIT_ATTN_SCORES
#if FEWBIT_ATTN_F16
cudaError_t launch_scores_f16(
#else
cudaError_t launch_scores_bf16(
#endif
    Kernel which, bool wide, const Params &p, unsigned grid, cudaStream_t st) {
    const bool biased = p.scores.slopes != nullptr || p.scores.bias != nullptr;
    if (biased) return wide ? launch_one<128, 2>(which, p, grid, st) : launch_one<64, 2>(which, p, grid, st);
    return wide ? launch_one<128, 1>(which, p, grid, st) : launch_one<64, 1>(which, p, grid, st);
}
#else
#if FEWBIT_ATTN_F16
cudaError_t launch_f16(
#else
cudaError_t launch_bf16(
#endif
    Kernel which, bool wide, const Params &p, unsigned grid, cudaStream_t st) {
    return wide ? launch_one<128, 0>(which, p, grid, st) : launch_one<64, 0>(which, p, grid, st);
}
#endif

}  // namespace attn
}  // namespace fewbit
