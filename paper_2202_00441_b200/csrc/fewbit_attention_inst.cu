// The attention kernels for one 16-bit type (FEWBIT_ATTN_F16: binary16, else bfloat16).
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

}  // namespace

#if FEWBIT_ATTN_F16
cudaError_t launch_f16(
#else
cudaError_t launch_bf16(
#endif
    Kernel which, bool wide, const Params &p, unsigned grid, cudaStream_t st) {
    switch (which) {
    case Kernel::forward:
        return wide ? launch<attention_fwd_kernel<T, 128>, fwd_smem<128>()>(p, grid * p.split, p.split, st) : launch<attention_fwd_kernel<T, 64>, fwd_smem<64>()>(p, grid * p.split, p.split, st);
    case Kernel::dq:
        return wide ? launch<attention_dq_kernel<T, 128>, dq_smem<128>()>(p, grid * p.split, p.split, st) : launch<attention_dq_kernel<T, 64>, dq_smem<64>()>(p, grid * p.split, p.split, st);
    default:
        return wide ? launch<attention_dkv_kernel<T, 128>, dkv_smem<128>()>(p, grid * p.split, p.split, st) : launch<attention_dkv_kernel<T, 64>, dkv_smem<64>()>(p, grid * p.split, p.split, st);
    }
}

}  // namespace attn
}  // namespace fewbit
