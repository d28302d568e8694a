// Launchers of the attention kernels, one set for each 16-bit type.
#pragma once
#include <cuda_runtime_api.h>

namespace fewbit {
namespace attn {
struct Params;
enum class Kernel { forward, dq, dkv, dkv_bias };   // dkv_bias: with the gradient of a bias by distance (launch_scores_* only)
// wide: head_dim above 64; grid: clusters of p.split CTAs
cudaError_t launch_bf16(Kernel which, bool wide, const Params &p, unsigned grid, cudaStream_t st);
cudaError_t launch_f16(Kernel which, bool wide, const Params &p, unsigned grid, cudaStream_t st);
// with caps, biases and masks (p.scores)
cudaError_t launch_scores_bf16(Kernel which, bool wide, const Params &p, unsigned grid, cudaStream_t st);
cudaError_t launch_scores_f16(Kernel which, bool wide, const Params &p, unsigned grid, cudaStream_t st);
// behind dkv_bias, with its Params: the sums by distance, heads x (2 * scores.reach + 1) (fewbit_bias.cu)
cudaError_t launch_bias_gradient(const Params &p, float *grad, cudaStream_t st);
}  // namespace attn
}  // namespace fewbit
