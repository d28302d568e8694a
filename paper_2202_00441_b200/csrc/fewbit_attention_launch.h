// Launchers of the attention kernels, one set for each 16-bit type.
#pragma once
#include <cuda_runtime_api.h>

namespace fewbit {
namespace attn {
struct Params;
enum class Kernel { forward, dq, dkv };
// wide: head_dim above 64; grid: clusters of p.split CTAs
cudaError_t launch_bf16(Kernel which, bool wide, const Params &p, unsigned grid, cudaStream_t st);
cudaError_t launch_f16(Kernel which, bool wide, const Params &p, unsigned grid, cudaStream_t st);
}  // namespace attn
}  // namespace fewbit
