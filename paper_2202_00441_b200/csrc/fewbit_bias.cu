// A learned bias of relative positions: the table by buckets spread over the distances, its gradient, and the gradient of a bias
// by distance from the sums that the dK and dV kernel left.
#include <limits>

#include "fewbit_attention.cuh"
#include "fewbit_attention_launch.h"

namespace fewbit {
bool pdl_enabled();

namespace attn {
namespace {

// ---------------------------------------------------------------------------------------------------
// the attention's gradient by distance
// ---------------------------------------------------------------------------------------------------
// A CTA takes 32 distances of one head, a lane each; its warps share the pairs of tiles.  Each pair of tiles holds a warp's sums
// over 32 x 32 pieces, 64 distances apiece; up to 8 of the 16 pieces have a given one.  The last CTA of a head adds up what
// lies at and beyond the table's ends.  No atomics: the order is fixed.
constexpr int kGradThreads = 1024, kGradWarps = kGradThreads / 32, kGradTogether = 4;

__global__ void __launch_bounds__(kGradThreads)
bias_gradient_kernel(Scores sc, int batch, int heads, int split, int groups, float *grad) {
    pdl_launch_dependents();
    __shared__ float part[2][kGradWarps][33];
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, head = blockIdx.y, tiles = sc.places, items = batch * tiles;
    pdl_wait();
    float *to = grad + static_cast<long long>(head) * (2 * sc.reach + 1) + sc.reach;   // of distance 0
    auto place_of = [&](int item) { return (static_cast<long long>(item / tiles) * heads + head) * tiles + item % tiles; };
    if (static_cast<int>(blockIdx.x) == groups) {
        float behind = 0.0f, ahead = 0.0f;
        for (long long i = threadIdx.x; i < static_cast<long long>(items) * split * 16; i += kGradThreads) {
            const long long place = place_of(static_cast<int>(i / (split * 16)));
            if (sc.written[place].w == 0) continue;
            const float2 v = reinterpret_cast<const float2 *>(sc.far + place * kFarFloats)[i % (split * 16)];
            behind += v.x;
            ahead += v.y;
        }
        part[0][warp][lane] = behind;
        part[1][warp][lane] = ahead;
        __syncthreads();
        if (warp < 2) {
            float sum = 0.0f;
            for (int k = 0; k < kGradWarps; ++k) sum += part[warp][k][lane];
            for (int o = 16; o > 0; o >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, o);
            if (lane == 0) to[warp == 0 ? -sc.reach : sc.reach] = sum;
        }
        return;
    }
    const int first = -sc.reach + 1 + 32 * static_cast<int>(blockIdx.x), d = first + lane;
    float sum = 0.0f;
    // up to 3 row tiles of a key tile have a pair at one of these distances; four such pairs of tiles wait for memory together
    for (long long at0 = warp; at0 < 3ll * items; at0 += kGradTogether * kGradWarps) {
        int4 written[kGradTogether];
        long long place[kGradTogether];
        int item[kGradTogether];
#pragma unroll
        for (int i = 0; i < kGradTogether; ++i) {
            item[i] = static_cast<int>(min((at0 + i * kGradWarps) / 3, items - 1ll));
            place[i] = place_of(item[i]);
            written[i] = sc.written[place[i]];
        }
#pragma unroll
        for (int i = 0; i < kGradTogether; ++i) {
            const long long at = at0 + i * kGradWarps;
            const int k0 = (written[i].w - 1) * kTile, reach = written[i].z, nearest = max(0, first_near(k0, reach, sc.reach));
            const int t = max(max(written[i].x, nearest), first_near(k0, reach, first + 32)) + static_cast<int>(at % 3);
            const bool there = at < 3ll * items && written[i].w > 0 && t < min(written[i].y, nearest + sc.near_tiles) && t * kTile <= k0 - reach + 127 - first;
            const float *from = sc.near + (place[i] * sc.near_tiles + (there ? t - nearest : 0)) * kNearFloats;
            const int u0 = d - (k0 - t * kTile - reach) + 32;         // in a piece on the diagonal
#pragma unroll
            for (int k = 0; k < 16; ++k) {
                const int u = u0 - 32 * (k & 3) + 32 * (k >> 2);
                sum += there && u >= 0 && u < 64 ? from[k * 64 + u] : 0.0f;
            }
        }
    }
    part[0][warp][lane] = sum;
    __syncthreads();
    if (warp == 0 && d < sc.reach) {
        sum = 0.0f;
        for (int k = 0; k < kGradWarps; ++k) sum += part[0][k][lane];
        to[d] = sum;
    }
}

}  // namespace

cudaError_t launch_bias_gradient(const Params &p, float *grad, cudaStream_t st) {
    const int groups = (2 * p.scores.reach - 1 + 31) / 32;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3(groups + 1, p.heads);
    cfg.blockDim = dim3(kGradThreads);
    cfg.stream = st;
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = attr;
    cfg.numAttrs = pdl_enabled() ? 1 : 0;
    return cudaLaunchKernelEx(&cfg, bias_gradient_kernel, p.scores, p.q_offsets != nullptr ? 1 : p.batch, p.heads, p.split, groups, grad);
}

}  // namespace attn

namespace {

// ---------------------------------------------------------------------------------------------------
// table by buckets <-> bias by distance
// ---------------------------------------------------------------------------------------------------
// A bucket of one direction is a run of distances: `start[b]` is its first one, for the exact buckets (start[b] = b) too.  The
// host finds the starts once for a call, and they travel as kernel parameters.
constexpr int kMaxBuckets = 1024;
struct Buckets {
    uint16_t start[kMaxBuckets + 1];  // start[n]: past every distance
    int n, both, reach;
};

__device__ __forceinline__ int bucket_of(const Buckets &b, int d) {
    const int n = b.both ? abs(d) : max(-d, 0);
    int low = 0, high = b.n;          // start[low] <= n < start[high]
    while (high - low > 1) {
        const int mid = (low + high) / 2;
        if (b.start[mid] <= n) low = mid;
        else high = mid;
    }
    return b.both && d > 0 ? low + b.n : low;
}

template <typename T>
__global__ void __launch_bounds__(256)
spread_kernel(const __grid_constant__ Buckets b, const T *table, int heads, float *bias) {
    pdl_launch_dependents();
    const int at = blockIdx.x * 256 + threadIdx.x;
    const int bucket = at <= 2 * b.reach ? bucket_of(b, at - b.reach) : 0;
    pdl_wait();
    if (at <= 2 * b.reach) bias[static_cast<long long>(blockIdx.y) * (2 * b.reach + 1) + at] = load1(table + static_cast<long long>(bucket) * heads + blockIdx.y);
}

// A warp adds up the distances of one bucket and head: lanes in turn, then the lanes.
template <typename T>
__global__ void __launch_bounds__(256)
gather_kernel(const __grid_constant__ Buckets b, const float *grad, int heads, T *table) {
    pdl_launch_dependents();
    const int bucket = blockIdx.x * 8 + (threadIdx.x >> 5), lane = threadIdx.x & 31;
    pdl_wait();
    if (bucket >= b.n * (b.both ? 2 : 1)) return;
    const float *mine = grad + static_cast<long long>(blockIdx.y) * (2 * b.reach + 1) + b.reach;   // of distance 0
    const bool ahead = bucket >= b.n;
    const int of = ahead ? bucket - b.n : bucket, first = b.start[of], end = min(static_cast<int>(b.start[of + 1]), b.reach + 1);
    float sum = 0.0f;
    for (int n = first + lane; n < end; n += 32)
        if (!ahead || n > 0) sum += mine[ahead ? n : -n];
    if (!b.both && of == 0)                                           // every key ahead of its row
        for (int n = 1 + lane; n <= b.reach; n += 32) sum += mine[n];
    for (int o = 16; o > 0; o >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, o);
    if (lane == 0) store1(table + static_cast<long long>(bucket) * heads + blockIdx.y, sum);
}

fewbit_status find_buckets(int buckets, int heads, int most, int both, fewbit_dtype dtype, Buckets *b) {
    if (!valid_dtype(dtype) || heads < 0 || buckets < (both ? 4 : 2) || buckets > kMaxBuckets || (both && buckets % 2) || most > FEWBIT_MAX_DISTANCE) return FEWBIT_ERR_INVALID_ARG;
    const int n = both ? buckets / 2 : buckets, exact = n / 2;
    if (most <= exact) return FEWBIT_ERR_INVALID_ARG;
    if (heads > 65535) return FEWBIT_ERR_TOO_LARGE;
    b->n = n;
    b->both = both != 0;
    b->reach = most;
    for (int i = 0; i <= exact; ++i) b->start[i] = static_cast<uint16_t>(i);
    // Bucket exact + i starts at the first distance d with (d / exact)^(n - exact) >= (most / exact)^i.  The two sides may be equal
    // (powers of two); their logarithms, of 64 bits and up to 8.4, then agree to 5e-19.  Of all sizes that are taken no other distance's comes
    // nearer to a border than 5.7e-16 (625 buckets to 3394, distance 1524; all of them were computed).
    static_assert(std::numeric_limits<long double>::digits >= 64);
    for (int i = 1; i < n - exact; ++i) {
        const long double border = logl(static_cast<long double>(exact)) + (logl(static_cast<long double>(most)) - logl(static_cast<long double>(exact))) * i / (n - exact);
        int d = b->start[exact + i - 1];
        while (d < most && logl(static_cast<long double>(d)) < border - 1e-16L) ++d;
        b->start[exact + i] = static_cast<uint16_t>(d);
    }
    b->start[n] = 65535;
    return FEWBIT_OK;
}

template <typename T>
cudaError_t spread(const Buckets &b, const void *table, int heads, float *bias, cudaStream_t st) {
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((2 * b.reach + 1 + 255) / 256, heads);
    cfg.blockDim = dim3(256);
    cfg.stream = st;
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = attr;
    cfg.numAttrs = pdl_enabled() ? 1 : 0;
    return cudaLaunchKernelEx(&cfg, spread_kernel<T>, b, static_cast<const T *>(table), heads, bias);
}
template <typename T>
cudaError_t gather(const Buckets &b, const float *grad, int heads, void *table, cudaStream_t st) {
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((b.n * (b.both ? 2 : 1) + 7) / 8, heads);
    cfg.blockDim = dim3(256);
    cfg.stream = st;
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = attr;
    cfg.numAttrs = pdl_enabled() ? 1 : 0;
    return cudaLaunchKernelEx(&cfg, gather_kernel<T>, b, grad, heads, static_cast<T *>(table));
}

fewbit_status cuda_status(cudaError_t err) {
    if (err == cudaSuccess) {
        g_launches.fetch_add(1, std::memory_order_relaxed);
        return FEWBIT_OK;
    }
    t_last_cuda_error = static_cast<int>(err);
    return FEWBIT_ERR_CUDA;
}

fewbit_status check_buffers(const void *table, const void *bias, fewbit_dtype dtype) {
    if (table == nullptr || bias == nullptr) return FEWBIT_ERR_INVALID_ARG;
    if (reinterpret_cast<uintptr_t>(table) % (dtype == FEWBIT_F32 ? 4 : 2) || reinterpret_cast<uintptr_t>(bias) % 4) return FEWBIT_ERR_ALIGNMENT;
    return FEWBIT_OK;
}

}  // namespace
}  // namespace fewbit

extern "C" {

fewbit_status fewbit_relative_bias_fwd(const void *table, int buckets, int heads, int max_distance, int bidirectional, fewbit_dtype dtype, float *bias, void *stream) {
    using namespace fewbit;
    Buckets b;
    if (const fewbit_status st = find_buckets(buckets, heads, max_distance, bidirectional, dtype, &b); st != FEWBIT_OK) return st;
    if (heads == 0) return FEWBIT_OK;
    if (const fewbit_status st = check_buffers(table, bias, dtype); st != FEWBIT_OK) return st;
    const cudaStream_t s = static_cast<cudaStream_t>(stream);
    return cuda_status(dtype == FEWBIT_F32 ? spread<float>(b, table, heads, bias, s) : dtype == FEWBIT_BF16 ? spread<__nv_bfloat16>(b, table, heads, bias, s) : spread<__half>(b, table, heads, bias, s));
}

fewbit_status fewbit_relative_bias_bwd(const float *grad, int buckets, int heads, int max_distance, int bidirectional, fewbit_dtype dtype, void *table, void *stream) {
    using namespace fewbit;
    Buckets b;
    if (const fewbit_status st = find_buckets(buckets, heads, max_distance, bidirectional, dtype, &b); st != FEWBIT_OK) return st;
    if (heads == 0) return FEWBIT_OK;
    if (const fewbit_status st = check_buffers(table, grad, dtype); st != FEWBIT_OK) return st;
    const cudaStream_t s = static_cast<cudaStream_t>(stream);
    return cuda_status(dtype == FEWBIT_F32 ? gather<float>(b, grad, heads, table, s) : dtype == FEWBIT_BF16 ? gather<__nv_bfloat16>(b, grad, heads, table, s) : gather<__half>(b, grad, heads, table, s));
}

}  // extern "C"
