// The residual stream of a transformer block: dropout of a branch and its addition (fewbit_dropout_*), and the RMS norm of
// the sum (fewbit_add_rms_norm_*).
//
// Mathematics, one row of n elements:
//   h = r + keep * x / (1 - p),  s = 1 / sqrt(mean(h^2) + eps),  u = h s,  y = u w
//   g = grad_y w:  grad_h' = grad_h + s (g - u mean(g u)),  grad_r = grad_h',  grad_x = keep * grad_h' / (1 - p),
//   grad_w = sum over rows of grad_y u
// with all of it in binary32; h is rounded when it is stored, and the norm takes the sum as it was before.  The mask is
// drawn from a counter (fewbit_random.cuh) in both directions and never stored; s is computed again.
#include <cuda_fp8.h>

#include <atomic>
#include <cmath>
#include <type_traits>

#include "fewbit_device.cuh"
#include "fewbit_random.cuh"

namespace fewbit {
bool pdl_enabled();
int device_sm_count(cudaError_t *err);

namespace {

fewbit_status cuda_status(cudaError_t err) {
    if (err == cudaSuccess) return FEWBIT_OK;
    t_last_cuda_error = static_cast<int>(err);
    return FEWBIT_ERR_CUDA;
}

// ---------------------------------------------------------------------------------------------------
// dropout
// ---------------------------------------------------------------------------------------------------
constexpr int kDropThreads = 256, kDropVectors = 4;          // pieces of 8 elements for each thread
constexpr int kDropElems = kDropThreads * kDropVectors * 8;

// Pieces of 8 elements at any element alignment: `wide` ones as vectors.
template <typename T>
__device__ __forceinline__ void load_piece(const T *p, float (&v)[8], long long left, bool wide) {
    if (wide && left >= 8) {
        load8(p, v, false);
        return;
    }
#pragma unroll
    for (int e = 0; e < 8; ++e) v[e] = e < left ? load1(p + e) : 0.0f;
}
template <typename T>
__device__ __forceinline__ void store_piece(T *p, const float (&v)[8], long long left, bool wide) {
    if (wide && left >= 8) {
        store8(p, v, false);
        return;
    }
#pragma unroll
    for (int e = 0; e < 8; ++e)
        if (e < left) store1(p + e, v[e]);
}

template <typename T, bool RESIDUAL>
__global__ void __launch_bounds__(kDropThreads)
dropout_kernel(const T *x, const T *residual, T *y, long long n, Drop d, bool wide) {
    pdl_launch_dependents();
    const long long first = static_cast<long long>(blockIdx.x) * kDropElems + threadIdx.x * 8;
    pdl_wait();
    float v[kDropVectors][8], r[kDropVectors][8];
#pragma unroll
    for (int i = 0; i < kDropVectors; ++i) {
        const long long at = first + i * (kDropThreads * 8);
        if (at >= n) break;
        load_piece(x + at, v[i], n - at, wide);
        if (RESIDUAL) load_piece(residual + at, r[i], n - at, wide);
    }
    const RandomKeys keys = random_keys(d);
#pragma unroll
    for (int i = 0; i < kDropVectors; ++i) {
        const long long at = first + i * (kDropThreads * 8);
        if (at >= n) break;
        if (d.on) drop<8>(d, keys, at, v[i]);
        if (RESIDUAL) {
#pragma unroll
            for (int e = 0; e < 8; ++e) v[i][e] += r[i][e];
        }
        store_piece(y + at, v[i], n - at, wide);
    }
}

fewbit_status check_drop(const fewbit_dropout_options *o, Drop *d) {
    if (o == nullptr || !(o->p >= 0.0) || !(o->p < 1.0)) return FEWBIT_ERR_INVALID_ARG;
    if (reinterpret_cast<uintptr_t>(o->seed_device) & 7) return FEWBIT_ERR_ALIGNMENT;
    const double limit = std::floor(o->p * 4294967296.0 + 0.5);
    d->seed = o->seed;
    d->seed_device = o->seed_device;
    d->place = o->place;
    d->limit = limit < 4294967295.0 ? static_cast<uint32_t>(limit) : 4294967295u;
    d->scale = static_cast<float>(1.0 / (1.0 - o->p));
    d->on = o->p > 0.0;
    return FEWBIT_OK;
}

template <typename T>
cudaError_t launch_dropout(const void *x, const void *residual, void *y, long long n, const Drop &d, bool wide, cudaStream_t st) {
    const unsigned grid = static_cast<unsigned>((n + kDropElems - 1) / kDropElems);
    const T *a = static_cast<const T *>(x), *r = static_cast<const T *>(residual);
    return residual != nullptr ? launch_pdl(dropout_kernel<T, true>, grid, kDropThreads, 0, st, pdl_enabled(), a, r, static_cast<T *>(y), n, d, wide)
                               : launch_pdl(dropout_kernel<T, false>, grid, kDropThreads, 0, st, pdl_enabled(), a, r, static_cast<T *>(y), n, d, wide);
}

fewbit_status dropout(const void *x, const void *residual, void *y, size_t n, fewbit_dtype dtype, const fewbit_dropout_options *o, void *stream) {
    Drop d;
    if (!valid_dtype(dtype)) return FEWBIT_ERR_INVALID_ARG;
    if (const fewbit_status st = check_drop(o, &d); st != FEWBIT_OK) return st;
    if (n == 0) return FEWBIT_OK;
    if (x == nullptr || y == nullptr) return FEWBIT_ERR_INVALID_ARG;
    if (n > static_cast<size_t>(INT32_MAX) * kDropElems) return FEWBIT_ERR_TOO_LARGE;
    const uintptr_t all = reinterpret_cast<uintptr_t>(x) | reinterpret_cast<uintptr_t>(residual) | reinterpret_cast<uintptr_t>(y);
    if (all & (dtype == FEWBIT_F32 ? 3 : 1)) return FEWBIT_ERR_ALIGNMENT;
    const bool wide = all % 16 == 0;
    const cudaStream_t s = static_cast<cudaStream_t>(stream);
    const long long m = static_cast<long long>(n);
    const cudaError_t err = dtype == FEWBIT_F32    ? launch_dropout<float>(x, residual, y, m, d, wide, s)
                            : dtype == FEWBIT_BF16 ? launch_dropout<__nv_bfloat16>(x, residual, y, m, d, wide, s)
                                                   : launch_dropout<__half>(x, residual, y, m, d, wide, s);
    if (err == cudaSuccess) g_launches.fetch_add(1, std::memory_order_relaxed);
    return cuda_status(err);
}

// ---------------------------------------------------------------------------------------------------
// norm of the residual stream
// ---------------------------------------------------------------------------------------------------
struct NormParams {
    const void *x, *residual;                                // forward: residual may be NULL
    const void *grad_y, *grad_h, *h_in;                      // backward: grad_h may be NULL
    const float *weight;                                     // NULL: ones
    void *h, *y;                                             // h may be NULL
    float *y_scale;
    void *grad_x, *grad_residual;                            // either may be NULL
    float *partial;                                          // weight gradient: a row of `width` sums for each group of threads
    Drop drop;
    long long rows;
    int width, group;                                        // group: threads of a row
    float eps, inv_width;
};

// N elements of a row for each thread, in pieces of V: piece i at column (i * group + thread) * V.
template <typename T, int V>
__device__ __forceinline__ void load_v(const T *p, float *v) {
    if constexpr (V == 8) {
        load8(p, *reinterpret_cast<float(*)[8]>(v), false);
    } else if constexpr (V == 4 && sizeof(T) == 4) {
        const float4 f = *reinterpret_cast<const float4 *>(p);
        v[0] = f.x; v[1] = f.y; v[2] = f.z; v[3] = f.w;
    } else if constexpr (V == 4) {
        const uint2 w = *reinterpret_cast<const uint2 *>(p);
        T e[4];
        memcpy(e, &w, 8);
#pragma unroll
        for (int i = 0; i < 4; ++i) v[i] = load1(&e[i]);
    } else {
        v[0] = load1(p);
    }
}
template <typename T, int V>
__device__ __forceinline__ void store_v(T *p, const float *v) {
    if constexpr (V == 8) {
        store8(p, *reinterpret_cast<const float(*)[8]>(v), false);
    } else if constexpr (V == 4 && sizeof(T) == 4) {
        *reinterpret_cast<float4 *>(p) = make_float4(v[0], v[1], v[2], v[3]);
    } else if constexpr (V == 4) {
        T e[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) store1(&e[i], v[i]);
        uint2 w;
        memcpy(&w, e, 8);
        *reinterpret_cast<uint2 *>(p) = w;
    } else {
        store1(p, v[0]);
    }
}
__device__ __forceinline__ void store_codes(uint8_t *p, const float *v, std::integral_constant<int, 1>) {
    *p = __nv_cvt_float_to_fp8(v[0], __NV_SATFINITE, __NV_E4M3);
}
template <int V>
__device__ __forceinline__ void store_codes(uint8_t *p, const float *v, std::integral_constant<int, V>) {
    uint32_t w[V / 4];
#pragma unroll
    for (int i = 0; i < V / 4; ++i) {
        const uint32_t lo = __nv_cvt_float2_to_fp8x2(make_float2(v[4 * i], v[4 * i + 1]), __NV_SATFINITE, __NV_E4M3);
        const uint32_t hi = __nv_cvt_float2_to_fp8x2(make_float2(v[4 * i + 2], v[4 * i + 3]), __NV_SATFINITE, __NV_E4M3);
        w[i] = lo | hi << 16;
    }
    if constexpr (V == 8) *reinterpret_cast<uint2 *>(p) = make_uint2(w[0], w[1]);
    else *reinterpret_cast<uint32_t *>(p) = w[0];
}
// The weight is any binary32 buffer: 4-byte aligned.
template <int V>
__device__ __forceinline__ void load_weight(const float *w, int col, float *v, bool wide) {
    if (w == nullptr) {
#pragma unroll
        for (int e = 0; e < V; ++e) v[e] = 1.0f;
    } else if (V >= 4 && wide) {
#pragma unroll
        for (int e = 0; e < V / 4; ++e) {
            const float4 f = __ldg(reinterpret_cast<const float4 *>(w + col) + e);
            v[4 * e] = f.x; v[4 * e + 1] = f.y; v[4 * e + 2] = f.z; v[4 * e + 3] = f.w;
        }
    } else {
#pragma unroll
        for (int e = 0; e < V; ++e) v[e] = __ldg(w + col + e);
    }
}
__device__ __forceinline__ float max_nan(float a, float b) {
    float d;
    asm("max.NaN.f32 %0, %1, %2;" : "=f"(d) : "f"(a), "f"(b));
    return d;
}

// Sums (or maxima) over the threads of a row, the same for all of them, in a fixed order.  `part` has 2 x 16 places and is
// read before the next barrier but one, so two of them in turn need no barrier of their own.
constexpr int kNormThreads = 512;                            // at most, in a CTA
template <bool MAX>
__device__ __forceinline__ float combine(float a, float b) { return MAX ? max_nan(a, b) : a + b; }
template <bool MAX, int K>
__device__ __forceinline__ void over_group(float (&v)[K], int group, float (*part)[16]) {
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) {
#pragma unroll
        for (int k = 0; k < K; ++k) v[k] = combine<MAX>(v[k], __shfl_xor_sync(0xffffffffu, v[k], o));
    }
    if (group == 32) return;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, warps = group >> 5, first = warp & ~(warps - 1);
    if (lane == 0) {
#pragma unroll
        for (int k = 0; k < K; ++k) part[k][warp] = v[k];
    }
    __syncthreads();
#pragma unroll
    for (int k = 0; k < K; ++k) v[k] = part[k][first + (lane & (warps - 1))];
    for (int o = warps >> 1; o > 0; o >>= 1) {
#pragma unroll
        for (int k = 0; k < K; ++k) v[k] = combine<MAX>(v[k], __shfl_xor_sync(0xffffffffu, v[k], o));
    }
}

template <typename T, int V, int N, bool CODES>
__global__ void __launch_bounds__(kNormThreads)
add_norm_fwd_kernel(const NormParams p) {
    pdl_launch_dependents();
    __shared__ float part[2][2][16];
    const int t = threadIdx.x & (p.group - 1);
    const long long row = static_cast<long long>(blockIdx.x) * (blockDim.x / p.group) + threadIdx.x / p.group;
    const bool live = row < p.rows;
    const long long at = (live ? row : 0) * p.width;
    const int width = live ? p.width : 0;
    pdl_wait();
    float h[N];
#pragma unroll
    for (int i = 0; i < N; i += V) {
        const int col = (i / V * p.group + t) * V;
        if (col < width) load_v<T, V>(static_cast<const T *>(p.x) + at + col, h + i);
    }
    float r[N];
    if (p.residual != nullptr) {
#pragma unroll
        for (int i = 0; i < N; i += V) {
            const int col = (i / V * p.group + t) * V;
            if (col < width) load_v<T, V>(static_cast<const T *>(p.residual) + at + col, r + i);
        }
    }
    if (p.drop.on) {
        const RandomKeys keys = random_keys(p.drop);
#pragma unroll
        for (int i = 0; i < N; i += V) {
            const int col = (i / V * p.group + t) * V;
            if (col < width) drop<V>(p.drop, keys, at + col, h + i);
        }
    }
    float sum[1] = {0.0f};
#pragma unroll
    for (int i = 0; i < N; i += V) {
        const int col = (i / V * p.group + t) * V;
        if (col >= width) break;
        if (p.residual != nullptr) {
#pragma unroll
            for (int e = 0; e < V; ++e) h[i + e] += r[i + e];
        }
        if (p.h != nullptr) store_v<T, V>(static_cast<T *>(p.h) + at + col, h + i);
#pragma unroll
        for (int e = 0; e < V; ++e) sum[0] = fmaf(h[i + e], h[i + e], sum[0]);
    }
    over_group<false>(sum, p.group, part[0]);
    const float s = rsqrtf(fmaf(sum[0], p.inv_width, p.eps));
    const bool wide = (reinterpret_cast<uintptr_t>(p.weight) & 15) == 0;
    float top[1] = {0.0f};
#pragma unroll
    for (int i = 0; i < N; i += V) {
        const int col = (i / V * p.group + t) * V;
        if (col >= width) break;
        float w[V];
        load_weight<V>(p.weight, col, w, wide);
#pragma unroll
        for (int e = 0; e < V; ++e) h[i + e] = h[i + e] * s * w[e];
        if constexpr (CODES) {
#pragma unroll
            for (int e = 0; e < V; ++e) top[0] = max_nan(top[0], fabsf(h[i + e]));
        } else {
            store_v<T, V>(static_cast<T *>(p.y) + at + col, h + i);
        }
    }
    if constexpr (CODES) {
        over_group<true>(top, p.group, part[1]);
        // a row that is not finite reads back as NaN, one too small for a scale as 0
        const bool fine = top[0] < INFINITY, some = top[0] >= 0x1p-117f;
        const float factor = fine && some ? 448.0f / top[0] : 0.0f;
        if (live && t == 0) p.y_scale[row] = !fine ? NAN : some ? top[0] / 448.0f : 0.0f;
#pragma unroll
        for (int i = 0; i < N; i += V) {
            const int col = (i / V * p.group + t) * V;
            if (col >= width) break;
#pragma unroll
            for (int e = 0; e < V; ++e) h[i + e] = fine && some ? h[i + e] * factor : 0.0f;
            store_codes(static_cast<uint8_t *>(p.y) + at + col, h + i, std::integral_constant<int, V>{});
        }
    }
}

template <typename T, int V, int N>
__global__ void __launch_bounds__(kNormThreads)
add_norm_bwd_kernel(const NormParams p) {
    pdl_launch_dependents();
    __shared__ float part[2][2][16];
    const int t = threadIdx.x & (p.group - 1), groups = blockDim.x / p.group, mine = threadIdx.x / p.group;
    pdl_wait();
    const bool wide = (reinterpret_cast<uintptr_t>(p.weight) & 15) == 0;
    RandomKeys keys;
    if (p.drop.on) keys = random_keys(p.drop);
    float dw[N];
#pragma unroll
    for (int i = 0; i < N; ++i) dw[i] = 0.0f;
    int turn = 0;
    for (long long base = static_cast<long long>(blockIdx.x) * groups; base < p.rows; base += static_cast<long long>(gridDim.x) * groups, turn ^= 1) {
        const long long row = base + mine;
        const bool live = row < p.rows;
        const long long at = (live ? row : 0) * p.width;
        const int width = live ? p.width : 0;
        float g[N], h[N];
#pragma unroll
        for (int i = 0; i < N; i += V) {
            const int col = (i / V * p.group + t) * V;
            if (col < width) {
                load_v<T, V>(static_cast<const T *>(p.grad_y) + at + col, g + i);
                load_v<T, V>(static_cast<const T *>(p.h_in) + at + col, h + i);
            }
        }
        float sums[2] = {0.0f, 0.0f};                        // of h^2 and of grad_y w h
#pragma unroll
        for (int i = 0; i < N; i += V) {
            const int col = (i / V * p.group + t) * V;
            if (col >= width) break;
            float w[V];
            load_weight<V>(p.weight, col, w, wide);
#pragma unroll
            for (int e = 0; e < V; ++e) {
                sums[0] = fmaf(h[i + e], h[i + e], sums[0]);
                sums[1] = fmaf(g[i + e] * w[e], h[i + e], sums[1]);
            }
        }
        over_group<false>(sums, p.group, part[turn]);
        const float s = rsqrtf(fmaf(sums[0], p.inv_width, p.eps));
        const float back = sums[1] * p.inv_width * s * s;
#pragma unroll
        for (int i = 0; i < N; i += V) {
            const int col = (i / V * p.group + t) * V;
            if (col >= width) break;
            float w[V], to[V];
            load_weight<V>(p.weight, col, w, wide);
            if (p.grad_h != nullptr) {
                load_v<T, V>(static_cast<const T *>(p.grad_h) + at + col, to);
            } else {
#pragma unroll
                for (int e = 0; e < V; ++e) to[e] = 0.0f;
            }
#pragma unroll
            for (int e = 0; e < V; ++e) {
                dw[i + e] = fmaf(g[i + e], h[i + e] * s, dw[i + e]);
                to[e] = fmaf(s, g[i + e] * w[e] - h[i + e] * back, to[e]);
            }
            if (p.grad_residual != nullptr) store_v<T, V>(static_cast<T *>(p.grad_residual) + at + col, to);
            if (p.grad_x != nullptr) {
                if (p.drop.on) drop<V>(p.drop, keys, at + col, to);
                store_v<T, V>(static_cast<T *>(p.grad_x) + at + col, to);
            }
        }
    }
    if (p.partial != nullptr) {
        float *to = p.partial + (static_cast<long long>(blockIdx.x) * groups + mine) * p.width;
#pragma unroll
        for (int i = 0; i < N; i += V) {
            const int col = (i / V * p.group + t) * V;
            if (col >= p.width) break;
#pragma unroll
            for (int e = 0; e < V; ++e) to[col + e] = dw[i + e];
        }
    }
}

// Adds up the groups' sums: 32 columns and 32 rows of threads for each CTA.
__global__ void __launch_bounds__(1024)
norm_weight_kernel(const float *partial, int rows, int width, float *to) {
    pdl_launch_dependents();
    __shared__ float part[32][33];
    const int lane = threadIdx.x & 31, row = threadIdx.x >> 5, col = blockIdx.x * 32 + lane;
    pdl_wait();
    float sum = 0.0f;
    if (col < width) {
#pragma unroll 8
        for (int c = row; c < rows; c += 32) sum += partial[static_cast<size_t>(c) * width + col];
    }
    part[row][lane] = sum;
    __syncthreads();
    sum = part[lane][row];                                   // transposed: a warp adds one column
    for (int o = 16; o > 0; o >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, o);
    if (lane == 0 && blockIdx.x * 32 + row < width) to[blockIdx.x * 32 + row] = sum;
}

constexpr int kNormMaxWidth = 16384;
constexpr int kNormCtas = 4;                                 // of 256 threads on an SM, backward

struct NormPlan {
    int v, n, group, threads;
};
// 16 elements a thread, 32 where a row would need more than 512 threads; narrow rows share a CTA of 256 threads.
NormPlan norm_plan(int64_t width, uintptr_t pointers, int elem) {
    NormPlan q;
    q.v = width % 8 == 0 && pointers % 16 == 0 ? 8 : width % 4 == 0 && pointers % (4 * elem) == 0 ? 4 : 1;
    q.n = width > 16 * kNormThreads ? 32 : 16;
    q.group = 32;
    while (q.group * q.n < width) q.group *= 2;
    q.threads = q.group < 256 ? 256 : q.group;
    return q;
}
// CTAs of the backward pass.
int64_t norm_ctas(int64_t rows, const NormPlan &q, int sms) {
    const int64_t per = q.threads / q.group, want = (rows + per - 1) / per, most = static_cast<int64_t>(sms) * kNormCtas * 256 / q.threads;
    return want < most ? want : most;
}

using NormLaunch = cudaError_t (*)(const NormParams &, unsigned, unsigned, cudaStream_t);
template <auto kernel>
cudaError_t launch_norm(const NormParams &p, unsigned grid, unsigned threads, cudaStream_t st) {
    return launch_pdl(kernel, grid, threads, 0, st, pdl_enabled(), p);
}
// [dtype][pieces of 8, 4, 1][16 or 32 elements a thread]
#define FEWBIT_NORM_ROW(T, K, ...) \
    {{launch_norm<K<T, 8, 16 __VA_ARGS__>>, launch_norm<K<T, 8, 32 __VA_ARGS__>>}, {launch_norm<K<T, 4, 16 __VA_ARGS__>>, launch_norm<K<T, 4, 32 __VA_ARGS__>>}, \
     {launch_norm<K<T, 1, 16 __VA_ARGS__>>, launch_norm<K<T, 1, 32 __VA_ARGS__>>}}
#define FEWBIT_COMMA ,
const NormLaunch kNormFwd[3][3][2] = {FEWBIT_NORM_ROW(float, add_norm_fwd_kernel, FEWBIT_COMMA false), FEWBIT_NORM_ROW(__nv_bfloat16, add_norm_fwd_kernel, FEWBIT_COMMA false),
                                      FEWBIT_NORM_ROW(__half, add_norm_fwd_kernel, FEWBIT_COMMA false)};
const NormLaunch kNormFwdCodes[3][3][2] = {FEWBIT_NORM_ROW(float, add_norm_fwd_kernel, FEWBIT_COMMA true), FEWBIT_NORM_ROW(__nv_bfloat16, add_norm_fwd_kernel, FEWBIT_COMMA true),
                                           FEWBIT_NORM_ROW(__half, add_norm_fwd_kernel, FEWBIT_COMMA true)};
const NormLaunch kNormBwd[3][3][2] = {FEWBIT_NORM_ROW(float, add_norm_bwd_kernel), FEWBIT_NORM_ROW(__nv_bfloat16, add_norm_bwd_kernel), FEWBIT_NORM_ROW(__half, add_norm_bwd_kernel)};
int piece_index(int v) { return v == 8 ? 0 : v == 4 ? 1 : 2; }

fewbit_status check_norm(const fewbit_norm_shape *s) {
    if (s == nullptr || !valid_dtype(s->dtype) || s->rows < 0 || s->width < 0 || !(s->eps >= 0) || !std::isfinite(s->eps)) return FEWBIT_ERR_INVALID_ARG;
    if (s->width > kNormMaxWidth) return FEWBIT_ERR_UNSUPPORTED;
    if (s->rows > INT32_MAX) return FEWBIT_ERR_TOO_LARGE;
    if (reinterpret_cast<uintptr_t>(s->weight) & 3) return FEWBIT_ERR_ALIGNMENT;
    return FEWBIT_OK;
}
NormParams norm_params(const fewbit_norm_shape *s, const Drop &d, const NormPlan &q) {
    NormParams p = {};
    p.weight = s->weight;
    p.drop = d;
    p.rows = s->rows;
    p.width = static_cast<int>(s->width);
    p.group = q.group;
    p.eps = s->eps;
    p.inv_width = 1.0f / static_cast<float>(s->width);
    return p;
}
uintptr_t bits_of(std::initializer_list<const void *> all) {
    uintptr_t x = 0;
    for (const void *p : all) x |= reinterpret_cast<uintptr_t>(p);
    return x;
}

}  // namespace
}  // namespace fewbit

extern "C" {

fewbit_status fewbit_dropout_fwd(const void *x, const void *residual, void *y, size_t n, fewbit_dtype dtype, const fewbit_dropout_options *options, void *stream) {
    return fewbit::dropout(x, residual, y, n, dtype, options, stream);
}

fewbit_status fewbit_dropout_bwd(const void *grad_out, void *grad_in, size_t n, fewbit_dtype dtype, const fewbit_dropout_options *options, void *stream) {
    return fewbit::dropout(grad_out, nullptr, grad_in, n, dtype, options, stream);
}

fewbit_status fewbit_add_rms_norm_fwd(const fewbit_norm_shape *s, const void *x, const void *residual, void *h, void *y, float *y_scale, int y_bits, void *stream) {
    using namespace fewbit;
    Drop d;
    if (const fewbit_status st = check_norm(s); st != FEWBIT_OK) return st;
    if (const fewbit_status st = check_drop(&s->dropout, &d); st != FEWBIT_OK) return st;
    if ((y_bits != 0 && y_bits != 8) || (y_bits == 0 && y_scale != nullptr) || (y_bits == 8 && s->rows > 0 && y_scale == nullptr)) return FEWBIT_ERR_INVALID_ARG;
    if (s->rows == 0) return FEWBIT_OK;
    const int elem = s->dtype == FEWBIT_F32 ? 4 : 2;
    if (s->width > 0 && (x == nullptr || y == nullptr)) return FEWBIT_ERR_INVALID_ARG;
    const uintptr_t of_type = bits_of({x, residual, h, y_bits == 8 ? nullptr : y});
    if (of_type % elem || reinterpret_cast<uintptr_t>(y_scale) % 4) return FEWBIT_ERR_ALIGNMENT;
    if (s->width == 0) return y_bits == 8 ? cuda_status(cudaMemsetAsync(y_scale, 0, s->rows * sizeof(float), static_cast<cudaStream_t>(stream))) : FEWBIT_OK;
    // codes take a byte an element: half or a quarter of the others' alignment is enough
    NormPlan q = norm_plan(s->width, of_type | (y_bits == 8 ? reinterpret_cast<uintptr_t>(y) * 2 : 0), elem);
    NormParams p = norm_params(s, d, q);
    p.x = x;
    p.residual = residual;
    p.h = h;
    p.y = y;
    p.y_scale = y_scale;
    const int64_t per = q.threads / q.group;
    const cudaError_t err = (y_bits == 8 ? kNormFwdCodes : kNormFwd)[s->dtype][piece_index(q.v)][q.n == 32](
        p, static_cast<unsigned>((s->rows + per - 1) / per), q.threads, static_cast<cudaStream_t>(stream));
    if (err == cudaSuccess) g_launches.fetch_add(1, std::memory_order_relaxed);
    return cuda_status(err);
}

size_t fewbit_add_rms_norm_workspace_bytes(const fewbit_norm_shape *s) {
    using namespace fewbit;
    if (check_norm(s) != FEWBIT_OK || s->rows == 0 || s->width == 0) return 0;
    cudaError_t err = cudaSuccess;
    const int sms = device_sm_count(&err);
    const NormPlan q = norm_plan(s->width, 0, 2);            // (the group does not depend on the alignment)
    return err != cudaSuccess ? 0 : static_cast<size_t>(norm_ctas(s->rows, q, sms)) * (q.threads / q.group) * s->width * sizeof(float);
}

fewbit_status fewbit_add_rms_norm_bwd(const fewbit_norm_shape *s, const void *grad_y, const void *grad_h, const void *h, void *grad_x, void *grad_residual,
                                      float *grad_weight, void *workspace, size_t workspace_bytes, void *stream) {
    using namespace fewbit;
    Drop d;
    if (const fewbit_status st = check_norm(s); st != FEWBIT_OK) return st;
    if (const fewbit_status st = check_drop(&s->dropout, &d); st != FEWBIT_OK) return st;
    const cudaStream_t stm = static_cast<cudaStream_t>(stream);
    const int elem = s->dtype == FEWBIT_F32 ? 4 : 2;
    const uintptr_t all = bits_of({grad_y, grad_h, h, grad_x, grad_residual});
    if (all % elem || reinterpret_cast<uintptr_t>(grad_weight) % 4 || reinterpret_cast<uintptr_t>(workspace) % 16) return FEWBIT_ERR_ALIGNMENT;
    if (s->width == 0 || (s->rows == 0 && grad_weight == nullptr)) return FEWBIT_OK;
    if (s->rows == 0) return cuda_status(cudaMemsetAsync(grad_weight, 0, s->width * sizeof(float), stm));   // the sum of nothing
    if (grad_y == nullptr || h == nullptr || (grad_weight != nullptr && workspace == nullptr)) return FEWBIT_ERR_INVALID_ARG;
    cudaError_t err = cudaSuccess;
    const int sms = device_sm_count(&err);
    if (err != cudaSuccess) return cuda_status(err);
    const NormPlan q = norm_plan(s->width, all, elem);
    const int64_t ctas = norm_ctas(s->rows, q, sms), groups = ctas * (q.threads / q.group);
    if (grad_weight != nullptr && workspace_bytes < static_cast<size_t>(groups) * s->width * sizeof(float)) return FEWBIT_ERR_ALLOC;
    NormParams p = norm_params(s, d, q);
    p.grad_y = grad_y;
    p.grad_h = grad_h;
    p.h_in = h;
    p.grad_x = grad_x;
    p.grad_residual = grad_residual;
    p.partial = grad_weight != nullptr ? static_cast<float *>(workspace) : nullptr;
    err = kNormBwd[s->dtype][piece_index(q.v)][q.n == 32](p, static_cast<unsigned>(ctas), q.threads, stm);
    if (err != cudaSuccess) return cuda_status(err);
    g_launches.fetch_add(1, std::memory_order_relaxed);
    if (grad_weight == nullptr) return FEWBIT_OK;
    err = launch_pdl(norm_weight_kernel, static_cast<unsigned>((s->width + 31) / 32), 1024, 0, stm, pdl_enabled(), static_cast<const float *>(p.partial),
                     static_cast<int>(groups), p.width, grad_weight);
    if (err == cudaSuccess) g_launches.fetch_add(1, std::memory_order_relaxed);
    return cuda_status(err);
}

}  // extern "C"
