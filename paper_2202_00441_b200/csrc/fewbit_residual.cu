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
#include "fewbit_packed.cuh"
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

// V neighbouring elements of 16 or 32 bits as they lie in memory.  Loads of several pieces are issued before the first is
// widened: a thread's loads then wait for memory together.
template <typename T, int V>
struct Piece {
    static constexpr int kBytes = V * static_cast<int>(sizeof(T)), kWords = kBytes < 4 ? 1 : kBytes / 4;
    uint32_t w[kWords];
    // `there`: else zeros
    __device__ __forceinline__ void load(const T *p, bool there = true) {
#pragma unroll
        for (int i = 0; i < kWords; ++i) w[i] = 0;
        if (!there) return;
        if constexpr (kBytes == 32) {
#pragma unroll
            for (int i = 0; i < kWords; i += 4) {
                const uint4 a = __ldcs(reinterpret_cast<const uint4 *>(p) + i / 4);
                w[i] = a.x; w[i + 1] = a.y; w[i + 2] = a.z; w[i + 3] = a.w;
            }
        } else if constexpr (kBytes == 16) {
            const uint4 a = __ldcs(reinterpret_cast<const uint4 *>(p));
            w[0] = a.x; w[1] = a.y; w[2] = a.z; w[3] = a.w;
        } else if constexpr (kBytes == 4) {
            w[0] = __ldcs(reinterpret_cast<const uint32_t *>(p));
        } else {
            w[0] = __ldcs(reinterpret_cast<const uint16_t *>(p));
        }
    }
    // A piece of 16 bytes to shared memory, and from there.  Of it, `left` elements are in the tensor.
    static __device__ __forceinline__ void copy(uint8_t *to, const T *p, long long left) {
        const uint32_t at = static_cast<uint32_t>(__cvta_generic_to_shared(to));
        const int bytes = static_cast<int>(min(left, static_cast<long long>(V))) * static_cast<int>(sizeof(T));
        asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" :: "r"(at), "l"(p), "r"(bytes) : "memory");
    }
    __device__ __forceinline__ void fetch(const uint8_t *from, bool there) {
        const uint4 a = there ? *reinterpret_cast<const uint4 *>(from) : make_uint4(0, 0, 0, 0);
        w[0] = a.x; w[1] = a.y; w[2] = a.z; w[3] = a.w;
    }
    __device__ __forceinline__ void widen(float *v) const {
#pragma unroll
        for (int e = 0; e < V; ++e) {
            if constexpr (sizeof(T) == 4) {
                v[e] = __uint_as_float(w[e]);
            } else {
                const uint16_t bits = static_cast<uint16_t>(w[e / 2] >> (16 * (e % 2)));
                T x;
                memcpy(&x, &bits, 2);
                v[e] = load1(&x);
            }
        }
    }
};

// ---------------------------------------------------------------------------------------------------
// dropout
// ---------------------------------------------------------------------------------------------------
// One pass: bound by memory with a residual (bfloat16, 16384 x 4096: 72 us = 5.6 TB/s, 86 % of a copy's rate), by the words without one
// (59 us, 69 %): four words take 18 products of 32 x 32 bits, which the multipliers do at a quarter of their rate, and 20 logic
// operations of half the issue rate.  A thread's loads are issued together: waiting for each as it is widened took twice as long.
constexpr int kDropThreads = 256, kDropVectors = 4;          // pieces of 8 elements for each thread
constexpr int kDropElems = kDropThreads * kDropVectors * 8;

template <typename T, bool RESIDUAL, bool HOST_SEED>
__global__ void __launch_bounds__(kDropThreads)
dropout_kernel(const T *x, const T *residual, T *y, long long n, const __grid_constant__ Drop d, bool wide) {
    pdl_launch_dependents();
    const long long first = static_cast<long long>(blockIdx.x) * kDropElems + threadIdx.x * 8;
    pdl_wait();
    const uint32_t high = static_cast<uint32_t>((static_cast<long long>(blockIdx.x) * kDropElems) >> 34);   // (a CTA's elements share it)
    if (wide && static_cast<long long>(blockIdx.x + 1) * kDropElems <= n) {
        Piece<T, 8> v[kDropVectors], r[kDropVectors];
#pragma unroll
        for (int i = 0; i < kDropVectors; ++i) {
            v[i].load(x + first + i * (kDropThreads * 8));
            if (RESIDUAL) r[i].load(residual + first + i * (kDropThreads * 8));
        }
        // (words first, while the loads are on their way: 16384 x 4096 with a residual 71.7 us, 73.6 otherwise; without one, where the
        // words themselves are the bound, 63.4 and 61.4)
        const RandomKeys keys = HOST_SEED ? d.keys : device_keys(d);
        uint32_t words[RESIDUAL ? kDropVectors : 1][8];
        auto draw_piece = [&](int i, uint32_t *w) { draw<8>(d, keys, static_cast<uint32_t>((first + i * (kDropThreads * 8)) >> 2), high, 0, w); };
        if (RESIDUAL && d.on) {
#pragma unroll
            for (int i = 0; i < kDropVectors; ++i) draw_piece(i, words[RESIDUAL ? i : 0]);
        }
        float f[kDropVectors][8];
#pragma unroll
        for (int i = 0; i < kDropVectors; ++i) v[i].widen(f[i]);
        if (d.on) {
#pragma unroll
            for (int i = 0; i < kDropVectors; ++i) {
                if (!RESIDUAL) draw_piece(i, words[0]);
                drop<8>(d, words[RESIDUAL ? i : 0], f[i]);
            }
        }
#pragma unroll
        for (int i = 0; i < kDropVectors; ++i) {
            if (RESIDUAL) {
                float g[8];
                r[i].widen(g);
#pragma unroll
                for (int e = 0; e < 8; e += 2) add2(f[i][e], f[i][e + 1], f[i][e], f[i][e + 1], g[e], g[e + 1]);
            }
            store8(y + first + i * (kDropThreads * 8), f[i], false);
        }
        return;
    }
    for (int i = 0; i < kDropVectors; ++i) {                 // the ragged end, or buffers of any alignment
        const long long at = first + i * (kDropThreads * 8);
        if (at >= n) return;
        const int valid = static_cast<int>(min(n - at, 8ll));
        float f[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) f[e] = e < valid ? load1(x + at + e) : 0.0f;
        if (d.on) {
            uint32_t words[8];
            draw<8>(d, HOST_SEED ? d.keys : device_keys(d), static_cast<uint32_t>(at >> 2), high, 0, words);
            drop<8>(d, words, f);
        }
#pragma unroll
        for (int e = 0; e < 8; ++e)
            if (e < valid) store1(y + at + e, RESIDUAL ? f[e] + load1(residual + at + e) : f[e]);
    }
}

fewbit_status check_drop(const fewbit_dropout_options *o, Drop *d) {
    if (o == nullptr || !(o->p >= 0.0) || !(o->p < 1.0)) return FEWBIT_ERR_INVALID_ARG;
    if (reinterpret_cast<uintptr_t>(o->seed_device) & 7) return FEWBIT_ERR_ALIGNMENT;
    const double limit = std::floor(o->p * 4294967296.0 + 0.5);
    d->seed = o->seed;
    d->seed_device = o->seed_device;
    d->keys = random_keys(o->seed);
    d->place = o->place;
    d->limit = limit < 4294967295.0 ? static_cast<uint32_t>(limit) : 4294967295u;
    d->scale = limit > 4294967295.0 ? 0.0f : static_cast<float>(1.0 / (1.0 - o->p));   // (no word is that large: the largest one passes, and counts 0)
    d->on = o->p > 0.0;
    return FEWBIT_OK;
}

template <typename T, bool RESIDUAL>
cudaError_t launch_dropout(const T *x, const T *residual, T *y, long long n, const Drop &d, bool wide, cudaStream_t st) {
    const unsigned grid = static_cast<unsigned>((n + kDropElems - 1) / kDropElems);
    return d.seed_device == nullptr ? launch_pdl(dropout_kernel<T, RESIDUAL, true>, grid, kDropThreads, 0, st, pdl_enabled(), x, residual, y, n, d, wide)
                                    : launch_pdl(dropout_kernel<T, RESIDUAL, false>, grid, kDropThreads, 0, st, pdl_enabled(), x, residual, y, n, d, wide);
}
template <typename T>
cudaError_t launch_dropout(const void *x, const void *residual, void *y, long long n, const Drop &d, bool wide, cudaStream_t st) {
    const T *a = static_cast<const T *>(x), *r = static_cast<const T *>(residual);
    return r != nullptr ? launch_dropout<T, true>(a, r, static_cast<T *>(y), n, d, wide, st) : launch_dropout<T, false>(a, r, static_cast<T *>(y), n, d, wide, st);
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
    float *partial;                                          // weight gradient: a row of `width` sums for each CTA
    Drop drop;
    long long rows;
    int width, group, per;                                   // group: threads of a row; per: rows in a CTA at a time
    int depth;                                               // backward: rows in shared memory at a time, 1 for none
    float eps, inv_width;
};

// N elements of a row for each thread, in pieces of V: piece i at column (i * group + thread) * V - lead, of which elements
// [lo, hi) are the row's.  LEAD: a row whose first element is not the first of an aligned piece of 16 bytes starts `lead` elements into
// one, so that rows of any width move in whole pieces but for their ends; what the ends' pieces hold of the rows beside it is
// replaced by zeros.  V 1: buffers of any alignment.
template <int V, bool LEAD>
struct Place {
    int col, lo, hi;
    __device__ __forceinline__ Place(int i, int group, int t, int lead, int width) {
        col = (i * group + t) * V - (LEAD ? lead : 0);
        lo = LEAD ? max(0, -col) : 0;
        hi = min(V, width - col);
    }
    __device__ __forceinline__ bool some() const { return hi > lo; }
    __device__ __forceinline__ bool whole() const { return LEAD ? lo == 0 && hi == V : true; }   // (if some)
    __device__ __forceinline__ void clear_others(float *v) const {
        if (LEAD && !(some() && whole())) {
#pragma unroll
            for (int e = 0; e < V; ++e) v[e] = e >= lo && e < hi ? v[e] : 0.0f;
        }
    }
};
// `left`: elements of the tensor from the piece's start on (LEAD: its last piece may reach past the end).
template <typename T, int V, bool LEAD>
__device__ __forceinline__ void load_place(Piece<T, V> &to, const T *row, const Place<V, LEAD> &at, long long left) {
    if (LEAD && left < V && at.some()) {
        uint8_t bytes[Piece<T, V>::kWords * 4] = {};
#pragma unroll
        for (int e = 0; e < V; ++e)
            if (e < left) memcpy(bytes + e * sizeof(T), row + at.col + e, sizeof(T));
        memcpy(to.w, bytes, sizeof(bytes));
    } else {
        to.load(row + at.col, at.some());
    }
}
template <typename T, int V, bool LEAD>
__device__ __forceinline__ void store_place(T *row, const Place<V, LEAD> &at, const float *v) {
    if (!at.some()) return;
    if constexpr (V > 1) {
        if (at.whole()) {
            if constexpr (V == 8) store8(row + at.col, *reinterpret_cast<const float(*)[8]>(v), false);
            else *reinterpret_cast<float4 *>(row + at.col) = make_float4(v[0], v[1], v[2], v[3]);
            return;
        }
    }
#pragma unroll
    for (int e = 0; e < V; ++e)
        if (e >= at.lo && e < at.hi) store1(row + at.col + e, v[e]);
}
template <int V, bool LEAD>
__device__ __forceinline__ void store_codes(uint8_t *row, const Place<V, LEAD> &at, const float *v) {
    if (!at.some()) return;
    if constexpr (V > 1) {
        if (at.whole()) {
            uint32_t w[V / 4];
#pragma unroll
            for (int i = 0; i < V / 4; ++i) {
                const uint32_t lo = __nv_cvt_float2_to_fp8x2(make_float2(v[4 * i], v[4 * i + 1]), __NV_SATFINITE, __NV_E4M3);
                const uint32_t hi = __nv_cvt_float2_to_fp8x2(make_float2(v[4 * i + 2], v[4 * i + 3]), __NV_SATFINITE, __NV_E4M3);
                w[i] = lo | hi << 16;
            }
            if constexpr (V == 8) *reinterpret_cast<uint2 *>(row + at.col) = make_uint2(w[0], w[1]);
            else *reinterpret_cast<uint32_t *>(row + at.col) = w[0];
            return;
        }
    }
#pragma unroll
    for (int e = 0; e < V; ++e)
        if (e >= at.lo && e < at.hi) row[at.col + e] = __nv_cvt_float_to_fp8(v[e], __NV_SATFINITE, __NV_E4M3);
}
// The weights of a thread's elements, 0 for others.  Any binary32 buffer, 4-byte aligned; `wide`: 16-byte aligned.
template <int V, int N, bool LEAD>
__device__ __forceinline__ void load_weights(const NormParams &p, int t, int lead, bool wide, float (&w)[N]) {
#pragma unroll
    for (int i = 0; i < N / V; ++i) {
        const Place<V, LEAD> at(i, p.group, t, lead, p.width);
        if (V > 1 && !LEAD && wide && p.weight != nullptr) {
#pragma unroll
            for (int e = 0; e < V; e += 4) {
                const float4 f = at.some() ? __ldg(reinterpret_cast<const float4 *>(p.weight + at.col) + e / 4) : make_float4(0.0f, 0.0f, 0.0f, 0.0f);
                w[i * V + e] = f.x; w[i * V + e + 1] = f.y; w[i * V + e + 2] = f.z; w[i * V + e + 3] = f.w;
            }
        } else {
#pragma unroll
            for (int e = 0; e < V; ++e) w[i * V + e] = e >= at.lo && e < at.hi ? (p.weight != nullptr ? __ldg(p.weight + at.col + e) : 1.0f) : 0.0f;
        }
    }
}
// use(i, words) for each piece of a thread's elements of the row that starts at element `at`.
template <int V, int N, bool LEAD, typename Use>
__device__ __forceinline__ void draw_row(const NormParams &p, int t, int lead, long long at, Use use) {
    const RandomKeys keys = device_keys(p.drop);
    const uint32_t high = static_cast<uint32_t>(at >> 34);
    auto go = [&](auto one_high) {
#pragma unroll
        for (int i = 0; i < N / V; ++i) {
            const long long first = at + Place<V, LEAD>(i, p.group, t, lead, p.width).col;
            uint32_t words[V];
            draw<V>(p.drop, keys, static_cast<uint32_t>(first >> 2), decltype(one_high)::value ? high : static_cast<uint32_t>(first >> 34), static_cast<uint32_t>(first) & 3, words);
            use(i, words);
        }
    };
    if (static_cast<uint32_t>((at + p.width) >> 34) == high) go(std::true_type{});
    else go(std::false_type{});                                       // a row in 2^34 elements
}
__device__ __forceinline__ float max_nan(float a, float b) {
    float d;
    asm("max.NaN.f32 %0, %1, %2;" : "=f"(d) : "f"(a), "f"(b));
    return d;
}

// Sums (or maxima) over the threads of a row, the same for all of them, in a fixed order.  A group of threads is a power of two
// up to a warp, or whole warps.  `part` has room for 16 warps and is read before the next barrier but one, so two of them in turn
// need no barrier of their own.
constexpr int kNormThreads = 512;                            // at most, in a CTA
template <bool MAX>
__device__ __forceinline__ float combine(float a, float b) { return MAX ? max_nan(a, b) : a + b; }
template <bool MAX, int K>
__device__ __forceinline__ void over_group(float (&v)[K], int group, float (*part)[16]) {
#pragma unroll
    for (int o = 1; o < 32; o *= 2) {
        if (o >= group) return;
#pragma unroll
        for (int k = 0; k < K; ++k) v[k] = combine<MAX>(v[k], __shfl_xor_sync(0xffffffffu, v[k], o));
    }
    if (group <= 32) return;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, warps = group >> 5, first = blockDim.x == group ? 0 : static_cast<int>(threadIdx.x) / group * warps;
    if (lane == 0) {
#pragma unroll
        for (int k = 0; k < K; ++k) part[k][warp] = v[k];
    }
    __syncthreads();
#pragma unroll
    for (int k = 0; k < K; ++k) v[k] = (lane & 15) < warps ? part[k][first + (lane & 15)] : 0.0f;   // (maxima are of magnitudes)
#pragma unroll
    for (int o = 8; o > 0; o >>= 1) {
#pragma unroll
        for (int k = 0; k < K; ++k) v[k] = combine<MAX>(v[k], __shfl_xor_sync(0xffffffffu, v[k], o));
    }
}

// Forward: a row for each group of threads, held in registers from its load to its results; one CTA's rows wait for memory while
// another's sums go round.  Bound by memory: bfloat16, 16384 x 4096, single passes, 88 us without dropout (93 % of a copy's rate), 100 with it (81 %:
// the words keep two thirds of the issue slots busy), 119 with 8-bit results; binary32 164 us (100 %).  Back to back the one with dropout takes 101 to 107 us.
// Places that are not the row's hold 0 from the load on, so that only loads and stores ask.
template <typename T, int V, bool LEAD, int N, bool CODES>
__global__ void __launch_bounds__(kNormThreads)
add_norm_fwd_kernel(const NormParams p) {
    pdl_launch_dependents();
    __shared__ float part[2][2][16];
    constexpr int P = N / V;
    using Of = Place<V, LEAD>;
    const int mine = p.per == 1 ? 0 : static_cast<int>(threadIdx.x) / p.group, t = static_cast<int>(threadIdx.x) - mine * p.group;
    const long long row = static_cast<long long>(blockIdx.x) * p.per + mine;
    const bool live = row < p.rows;
    const long long at = (live ? row : 0) * p.width, left = p.rows * p.width - at;
    const int width = live ? p.width : 0, lead = LEAD ? static_cast<int>(at & (V - 1)) : 0;
    pdl_wait();
    float h[N];
    {
        Piece<T, V> x[P], r[P];
#pragma unroll
        for (int i = 0; i < P; ++i) {
            const Of o(i, p.group, t, lead, width);
            load_place(x[i], static_cast<const T *>(p.x) + at, o, left - o.col);
        }
        if (p.residual != nullptr) {
#pragma unroll
            for (int i = 0; i < P; ++i) {
                const Of o(i, p.group, t, lead, width);
                load_place(r[i], static_cast<const T *>(p.residual) + at, o, left - o.col);
            }
        }
        uint32_t words[N];
        if (p.drop.on) {                                              // while the loads are on their way
            draw_row<V, N, LEAD>(p, t, lead, at, [&](int i, const uint32_t(&w)[V]) {
#pragma unroll
                for (int e = 0; e < V; ++e) words[i * V + e] = w[e];
            });
        }
#pragma unroll
        for (int i = 0; i < P; ++i) x[i].widen(h + i * V);
        if (p.drop.on) drop<N>(p.drop, words, h);
        if (p.residual != nullptr) {
            float f[N];
#pragma unroll
            for (int i = 0; i < P; ++i) r[i].widen(f + i * V);
#pragma unroll
            for (int i = 0; i < N; i += 2) add2(h[i], h[i + 1], h[i], h[i + 1], f[i], f[i + 1]);
        }
    }
#pragma unroll
    for (int i = 0; i < P; ++i) {
        const Of o(i, p.group, t, lead, width);
        o.clear_others(h + i * V);
        if (p.h != nullptr) store_place(static_cast<T *>(p.h) + at, o, h + i * V);
    }
    float two[2] = {0.0f, 0.0f};
#pragma unroll
    for (int i = 0; i < N; i += 2) fma2(two[0], two[1], h[i], h[i + 1], h[i], h[i + 1], two[0], two[1]);
    float sum[1] = {two[0] + two[1]};
    float w[N];
    load_weights<V, N, LEAD>(p, t, lead, (reinterpret_cast<uintptr_t>(p.weight) & 15) == 0, w);
    over_group<false>(sum, p.group, part[0]);
    const float s = rsqrtf(fmaf(sum[0], p.inv_width, p.eps));
#pragma unroll
    for (int i = 0; i < N; i += 2) {
        mul2(h[i], h[i + 1], h[i], h[i + 1], s, s);
        mul2(h[i], h[i + 1], h[i], h[i + 1], w[i], w[i + 1]);
    }
    if constexpr (!CODES) {
#pragma unroll
        for (int i = 0; i < P; ++i) store_place(static_cast<T *>(p.y) + at, Of(i, p.group, t, lead, width), h + i * V);
    } else {
        float top[1] = {0.0f};
#pragma unroll
        for (int i = 0; i < P; ++i) {
            const Of o(i, p.group, t, lead, width);
#pragma unroll
            for (int e = 0; e < V; ++e)                               // (0 times the factor of a row that is not finite is not 0)
                if (e >= o.lo && e < o.hi) top[0] = max_nan(top[0], fabsf(h[i * V + e]));
        }
        over_group<true>(top, p.group, part[1]);
        // a row that is not finite reads back as NaN, one too small for a scale as 0
        const bool fine = top[0] < INFINITY, some = top[0] >= 0x1p-117f;
        const float factor = fine && some ? 448.0f / top[0] : 0.0f;
        if (live && t == 0) p.y_scale[row] = !fine ? NAN : some ? top[0] / 448.0f : 0.0f;
#pragma unroll
        for (int i = 0; i < P; ++i) {
#pragma unroll
            for (int e = 0; e < V; ++e) h[i * V + e] = fine && some ? h[i * V + e] * factor : 0.0f;
            store_codes(static_cast<uint8_t *>(p.y) + at, Of(i, p.group, t, lead, width), h + i * V);
        }
    }
}

// Backward: CTAs stay and take rows in turn, so that the weight's gradient is summed in registers.  bfloat16, 16384 x 4096: 97 us without
// dropout (84 % of a copy's rate), 149 with it (69 %: no unit is at its limit, issue 60 %, memory two thirds; the words come when a row's
// loads have been used, and 16 warps an SM leave their chain uncovered); binary32 177 us (92 %).  Two CTAs of 256 threads that hold the weights beat three that read them again for
// every row (95 and 134 us), and words drawn in front of the sums (149 and 159).
// AHEAD: each thread copies its pieces of the next rows to places of its own in shared memory, `depth` - 1 rows ahead of their use
// (pieces of 16 bytes), so that a few CTAs keep memory busy while their rows' sums go round.
template <typename T, int V, bool LEAD, int N, int THREADS, int CTAS, bool AHEAD>
__global__ void __launch_bounds__(THREADS, CTAS)
add_norm_bwd_kernel(const NormParams p) {
    pdl_launch_dependents();
    extern __shared__ __align__(16) uint8_t ahead[];
    __shared__ float part[2][2][16];
    constexpr int P = N / V;
    using Of = Place<V, LEAD>;
    using Data = Piece<T, V>;
    const int groups = p.per, mine = groups == 1 ? 0 : static_cast<int>(threadIdx.x) / p.group, t = static_cast<int>(threadIdx.x) - mine * p.group;
    const long long stride = static_cast<long long>(gridDim.x) * groups;
    const int rounds = static_cast<int>((p.rows - static_cast<long long>(blockIdx.x) * groups + stride - 1) / stride);
    const T *const from[3] = {static_cast<const T *>(p.grad_y), static_cast<const T *>(p.h_in), static_cast<const T *>(p.grad_h)};
    auto row_of = [&](int round) { return round * stride + static_cast<long long>(blockIdx.x) * groups + mine; };
    auto place = [&](int stage, int a, int i) { return ahead + ((stage * 3 + a) * P + i) * (THREADS * 16) + threadIdx.x * 16; };
    auto lead_of = [&](long long at) { return LEAD ? static_cast<int>(at & (V - 1)) : 0; };
    auto copy = [&](int round, int stage) {
        if constexpr (AHEAD) {
            const long long row = row_of(round);
            if (round < rounds && row < p.rows) {
                const long long at = row * p.width, left = p.rows * p.width - at;
#pragma unroll
                for (int a = 0; a < 3; ++a) {
                    if (a == 2 && p.grad_h == nullptr) break;
#pragma unroll
                    for (int i = 0; i < P; ++i) {
                        const Of o(i, p.group, t, lead_of(at), p.width);
                        if (o.some()) Data::copy(place(stage, a, i), from[a] + at + o.col, LEAD ? left - o.col : V);
                    }
                }
            }
            asm volatile("cp.async.commit_group;" ::: "memory");
        }
    };
    pdl_wait();
    const bool wide = (reinterpret_cast<uintptr_t>(p.weight) & 15) == 0;
    // (LEAD: a group's rows all start as far into a piece, see norm_ctas)
    float dw[N], w[N];
    if constexpr (AHEAD) load_weights<V, N, LEAD>(p, t, lead_of((static_cast<long long>(blockIdx.x) * groups + mine) * p.width), wide, w);
#pragma unroll
    for (int i = 0; i < N; ++i) dw[i] = 0.0f;
    for (int r = 0; r + 1 < p.depth; ++r) copy(r, r);
    int stage = 0;
    for (int round = 0; round < rounds; ++round) {
        const long long row = row_of(round), at = (row < p.rows ? row : 0) * p.width;
        const bool live = row < p.rows;
        const int lead = lead_of(at);
        float g[N], h[N];
        [[maybe_unused]] Data more[AHEAD ? 1 : P];           // of grad_h
        if constexpr (AHEAD) {
            copy(round + p.depth - 1, stage == 0 ? p.depth - 1 : stage - 1);
            if (p.depth == 3) asm volatile("cp.async.wait_group 2;" ::: "memory");
            else asm volatile("cp.async.wait_group 1;" ::: "memory");
#pragma unroll
            for (int i = 0; i < P; ++i) {
                Data a, b;
                const Of o(i, p.group, t, lead, p.width);
                a.fetch(place(stage, 0, i), live && o.some());
                b.fetch(place(stage, 1, i), live && o.some());
                a.widen(g + i * V);
                b.widen(h + i * V);
                o.clear_others(g + i * V);
                o.clear_others(h + i * V);
            }
        } else {
            const long long left = p.rows * p.width - at;
            Data a[P], b[P];
#pragma unroll
            for (int i = 0; i < P; ++i) {
                const Of o(i, p.group, t, lead, live ? p.width : -8);
                load_place(a[i], from[0] + at, o, left - o.col);
                load_place(b[i], from[1] + at, o, left - o.col);
                if (p.grad_h != nullptr) load_place(more[i], from[2] + at, o, left - o.col);
            }
#pragma unroll
            for (int i = 0; i < P; ++i) {
                const Of o(i, p.group, t, lead, live ? p.width : -8);
                a[i].widen(g + i * V);
                b[i].widen(h + i * V);
                o.clear_others(g + i * V);
                o.clear_others(h + i * V);
            }
        }
        float sums[2];                                       // of h^2 and of grad_y w h
        {
            float hh[2] = {0.0f, 0.0f}, gh[2] = {0.0f, 0.0f};
            if constexpr (!AHEAD) load_weights<V, N, LEAD>(p, t, lead, wide, w);
#pragma unroll
            for (int i = 0; i < N; i += 2) {
                float a, b;
                fma2(hh[0], hh[1], h[i], h[i + 1], h[i], h[i + 1], hh[0], hh[1]);
                mul2(a, b, g[i], g[i + 1], w[i], w[i + 1]);
                fma2(gh[0], gh[1], a, b, h[i], h[i + 1], gh[0], gh[1]);
            }
            sums[0] = hh[0] + hh[1];
            sums[1] = gh[0] + gh[1];
        }
        over_group<false>(sums, p.group, part[round & 1]);
        const float s = live ? rsqrtf(fmaf(sums[0], p.inv_width, p.eps)) : 0.0f;   // (no row, and eps 0: infinite, and 0 times it the weights' sums)
        const float back = -sums[1] * p.inv_width * s * s;
        if constexpr (!AHEAD) load_weights<V, N, LEAD>(p, t, lead, wide, w);
#pragma unroll
        for (int i = 0; i < N; i += 2) {                     // g becomes s (g w - h back), dw takes g h s
            float a, b;
            mul2(a, b, h[i], h[i + 1], s, s);
            fma2(dw[i], dw[i + 1], g[i], g[i + 1], a, b, dw[i], dw[i + 1]);
            mul2(g[i], g[i + 1], g[i], g[i + 1], w[i], w[i + 1]);
            fma2(g[i], g[i + 1], h[i], h[i + 1], back, back, g[i], g[i + 1]);
        }
        if (p.grad_h != nullptr) {
#pragma unroll
            for (int i = 0; i < P; ++i) {
                if constexpr (AHEAD) {
                    Data c;
                    c.fetch(place(stage, 2, i), live && Of(i, p.group, t, lead, p.width).some());
                    c.widen(h + i * V);
                } else {
                    more[i].widen(h + i * V);
                }
            }
#pragma unroll
            for (int i = 0; i < N; i += 2) fma2(g[i], g[i + 1], g[i], g[i + 1], s, s, h[i], h[i + 1]);
        } else {
#pragma unroll
            for (int i = 0; i < N; i += 2) mul2(g[i], g[i + 1], g[i], g[i + 1], s, s);
        }
        if (p.grad_residual != nullptr && live) {
#pragma unroll
            for (int i = 0; i < P; ++i) store_place(static_cast<T *>(p.grad_residual) + at, Of(i, p.group, t, lead, p.width), g + i * V);
        }
        if (p.grad_x != nullptr && live) {
            if (p.drop.on) draw_row<V, N, LEAD>(p, t, lead, at, [&](int i, const uint32_t(&w)[V]) { drop<V>(p.drop, w, g + i * V); });
#pragma unroll
            for (int i = 0; i < P; ++i) store_place(static_cast<T *>(p.grad_x) + at, Of(i, p.group, t, lead, p.width), g + i * V);
        }
        stage = stage + 1 == p.depth ? 0 : stage + 1;
    }
    if (p.partial != nullptr) {
        // (LEAD: a group's rows all start as far into a piece, see norm_ctas)
        const int lead = lead_of((static_cast<long long>(blockIdx.x) * groups + mine) * p.width);
        float *to = p.partial + static_cast<long long>(blockIdx.x) * p.width;
        float *sums = reinterpret_cast<float *>(ahead) + mine * p.width;   // several groups: [group][column] in shared memory first
        if (groups > 1) {
            if constexpr (AHEAD) asm volatile("cp.async.wait_all;" ::: "memory");
            __syncthreads();
        }
#pragma unroll
        for (int i = 0; i < P; ++i) {
            const Of o(i, p.group, t, lead, p.width);
#pragma unroll
            for (int e = 0; e < V; ++e)
                if (e >= o.lo && e < o.hi) (groups > 1 ? sums : to)[o.col + e] = dw[i * V + e];
        }
        if (groups > 1) {
            __syncthreads();
            for (int c = threadIdx.x; c < p.width; c += blockDim.x) {
                float sum = 0.0f;
                for (int k = 0; k < groups; ++k) sum += reinterpret_cast<const float *>(ahead)[k * p.width + c];
                to[c] = sum;
            }
        }
    }
}

// Adds up the CTAs' sums: 32 columns and 32 rows of threads for each CTA.
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

enum { kWhole, kLead, kSingle };                             // pieces of 16 bytes that are whole, or not at the rows' ends (rows of 4099: 1.5 to 2 times as long); single elements (4 to 8 times)
struct NormPlan {
    int kind, n, group, threads;
};
// 16 elements a thread; 32 where a row would need more than 512 threads, 8 where a warp's part holds it.  Rows of up to 128
// threads share a CTA.
NormPlan norm_plan(int64_t width, uintptr_t pointers, int elem) {
    NormPlan q;
    q.kind = pointers % 16 != 0 ? kSingle : width % (16 / elem) == 0 ? kWhole : kLead;
    int span = static_cast<int>(q.kind == kLead ? width + 16 / elem - 1 : width);
    if (span > kNormMaxWidth) {
        q.kind = kSingle;
        span = static_cast<int>(width);
    }
    q.n = span > 16 * kNormThreads ? 32 : span <= 256 ? 8 : 16;
    q.group = 1;
    while (q.group < 32 && q.group * q.n < span) q.group *= 2;
    if (q.group * q.n < span) q.group = (span + q.n * 32 - 1) / (q.n * 32) * 32;
    q.threads = q.group > 128 ? q.group : 256 / q.group * q.group;
    return q;
}
// CTAs of the backward pass: as many as fit at once.  With kLead, groups of threads that take several rows take every 8th one, or
// a multiple of 8: then the same elements of each.
// Rows that a CTA of 512 threads holds, but none of 256: its sums are the weight's gradient without a second launch (5 rows of 640
// elements: 9.0 us with two CTAs, 7.7 so).  Rows that it would have to take in turn come sooner from several CTAs (4 rows of 4096: 10.3
// us, 12.2 from one).
void widen_plan(int64_t rows, NormPlan *q) {
    if (q->n == 16 && q->group <= 128 && rows > 256 / q->group && rows <= 512 / q->group) q->threads = 512 / q->group * q->group;
}
constexpr bool norm_ahead(int kind, int elem, int n) { return kind != kSingle && elem * n < 128; }
constexpr int norm_ctas_on_sm(bool ahead, int n, int threads) { return threads > 256 ? 1 : ahead && n == 16 ? 2 : 3; }
int64_t norm_ctas(int64_t rows, const NormPlan &q, int elem, int sms) {
    const int64_t per = q.threads / q.group, want = (rows + per - 1) / per;
    int64_t most = static_cast<int64_t>(sms) * norm_ctas_on_sm(norm_ahead(q.kind, elem, q.n), q.n, q.threads);
    if (q.kind == kLead) most = most < 8 ? 8 : most / 8 * 8;
    return want < most ? want : most;
}

using NormLaunch = cudaError_t (*)(NormParams &, unsigned, unsigned, cudaStream_t);
template <auto kernel>
cudaError_t launch_fwd(NormParams &p, unsigned grid, unsigned threads, cudaStream_t st) {
    return launch_pdl(kernel, grid, threads, 0, st, pdl_enabled(), p);
}
template <typename T, int V, bool LEAD, int N, int THREADS>
cudaError_t launch_bwd(NormParams &p, unsigned grid, unsigned threads, cudaStream_t st) {
    constexpr bool kAhead = norm_ahead(V == 1 ? kSingle : kWhole, sizeof(T), N);
    constexpr int kStage = 3 * N * static_cast<int>(sizeof(T)) * THREADS, kCtas = norm_ctas_on_sm(kAhead, N, THREADS), kRoom = 225 * 1024 / kCtas;
    constexpr int kDepth = !kAhead ? 1 : 3 * kStage <= kRoom ? 3 : 2;
    static_assert(!kAhead || kDepth * kStage <= kRoom);
    constexpr int kSums = 4 * N * THREADS, kShared = kDepth > 1 && kDepth * kStage > kSums ? kDepth * kStage : kSums;
    constexpr auto kernel = add_norm_bwd_kernel<T, V, LEAD, N, THREADS, kCtas, (kDepth > 1)>;
    p.depth = kDepth;
    if constexpr (kShared > 32 * 1024) {
        static std::atomic<unsigned long long> ready{0};              // devices (up to 64) whose limit has been raised
        int dev = 0;
        cudaError_t err = cudaGetDevice(&dev);
        if (err != cudaSuccess) return err;
        const unsigned long long bit = dev < 64 ? 1ull << dev : 0;
        if ((ready.load(std::memory_order_relaxed) & bit) == 0) {
            err = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, kShared);
            if (err != cudaSuccess) return err;
            ready.fetch_or(bit, std::memory_order_relaxed);
        }
    }
    return launch_pdl(kernel, grid, threads, kShared, st, pdl_enabled(), p);
}
// [dtype][kind][8, 16 or 32 elements a thread]
#define FEWBIT_NORM_KIND(T, V, LEAD, CODES) \
    {launch_fwd<add_norm_fwd_kernel<T, V, LEAD, 8, CODES>>, launch_fwd<add_norm_fwd_kernel<T, V, LEAD, 16, CODES>>, launch_fwd<add_norm_fwd_kernel<T, V, LEAD, 32, CODES>>}
#define FEWBIT_NORM_FWD(T, CODES) {FEWBIT_NORM_KIND(T, 16 / sizeof(T), false, CODES), FEWBIT_NORM_KIND(T, 16 / sizeof(T), true, CODES), FEWBIT_NORM_KIND(T, 1, false, CODES)}
const NormLaunch kNormFwd[3][3][3] = {FEWBIT_NORM_FWD(float, false), FEWBIT_NORM_FWD(__nv_bfloat16, false), FEWBIT_NORM_FWD(__half, false)};
const NormLaunch kNormFwdCodes[3][3][3] = {FEWBIT_NORM_FWD(float, true), FEWBIT_NORM_FWD(__nv_bfloat16, true), FEWBIT_NORM_FWD(__half, true)};
int size_index(const NormPlan &q) { return q.n == 8 ? 0 : q.n == 16 ? 1 : 2; }
// [dtype][kind][up to 256 threads of 8, of 16, up to 512 of 16, of 32]
#define FEWBIT_NORM_SIZES(T, V, LEAD) {launch_bwd<T, V, LEAD, 8, 256>, launch_bwd<T, V, LEAD, 16, 256>, launch_bwd<T, V, LEAD, 16, 512>, launch_bwd<T, V, LEAD, 32, 512>}
#define FEWBIT_NORM_BWD(T) {FEWBIT_NORM_SIZES(T, 16 / sizeof(T), false), FEWBIT_NORM_SIZES(T, 16 / sizeof(T), true), FEWBIT_NORM_SIZES(T, 1, false)}
const NormLaunch kNormBwd[3][3][4] = {FEWBIT_NORM_BWD(float), FEWBIT_NORM_BWD(__nv_bfloat16), FEWBIT_NORM_BWD(__half)};

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
    p.per = q.threads / q.group;
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
    // codes take a byte an element: a half or a quarter of the others' alignment is enough
    NormPlan q = norm_plan(s->width, of_type | (y_bits == 8 ? reinterpret_cast<uintptr_t>(y) * elem : 0), elem);
    NormParams p = norm_params(s, d, q);
    p.x = x;
    p.residual = residual;
    p.h = h;
    p.y = y;
    p.y_scale = y_scale;
    const int64_t per = q.threads / q.group;
    const cudaError_t err = (y_bits == 8 ? kNormFwdCodes : kNormFwd)[s->dtype][q.kind][size_index(q)](
        p, static_cast<unsigned>((s->rows + per - 1) / per), q.threads, static_cast<cudaStream_t>(stream));
    if (err == cudaSuccess) g_launches.fetch_add(1, std::memory_order_relaxed);
    return cuda_status(err);
}

size_t fewbit_add_rms_norm_workspace_bytes(const fewbit_norm_shape *s) {
    using namespace fewbit;
    if (check_norm(s) != FEWBIT_OK || s->rows == 0 || s->width == 0) return 0;
    cudaError_t err = cudaSuccess;
    const int sms = device_sm_count(&err);
    size_t most = 0;
    for (uintptr_t pointers : {0, 1}) {                      // (buffers of any alignment)
        NormPlan q = norm_plan(s->width, pointers, s->dtype == FEWBIT_F32 ? 4 : 2);
        widen_plan(s->rows, &q);
        const size_t bytes = static_cast<size_t>(norm_ctas(s->rows, q, s->dtype == FEWBIT_F32 ? 4 : 2, sms)) * s->width * sizeof(float);
        if (bytes > most) most = bytes;
    }
    return err != cudaSuccess ? 0 : most;
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
    NormPlan q = norm_plan(s->width, all, elem);
    widen_plan(s->rows, &q);
    const int64_t ctas = norm_ctas(s->rows, q, elem, sms);
    if (grad_weight != nullptr && workspace_bytes < static_cast<size_t>(ctas) * s->width * sizeof(float)) return FEWBIT_ERR_ALLOC;
    NormParams p = norm_params(s, d, q);
    p.grad_y = grad_y;
    p.grad_h = grad_h;
    p.h_in = h;
    p.grad_x = grad_x;
    p.grad_residual = grad_residual;
    p.partial = grad_weight != nullptr && ctas > 1 ? static_cast<float *>(workspace) : grad_weight;
    err = kNormBwd[s->dtype][q.kind][q.threads <= 256 ? size_index(q) : 1 + size_index(q)](p, static_cast<unsigned>(ctas), q.threads, stm);
    if (err != cudaSuccess) return cuda_status(err);
    g_launches.fetch_add(1, std::memory_order_relaxed);
    if (grad_weight == nullptr || ctas == 1) return FEWBIT_OK;
    err = launch_pdl(norm_weight_kernel, static_cast<unsigned>((s->width + 31) / 32), 1024, 0, stm, pdl_enabled(), static_cast<const float *>(p.partial),
                     static_cast<int>(ctas), p.width, grad_weight);
    if (err == cudaSuccess) g_launches.fetch_add(1, std::memory_order_relaxed);
    return cuda_status(err);
}

}  // extern "C"
