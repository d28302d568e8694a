// One AdamW step over many tensors (fewbit_adamw_step): moments in binary32, or in 8 bits with one
// scale for each block of 256 elements.
//
// Mathematics: the four lines of the header's formula per element; in 8 bits the block's largest
// magnitude before the codes.  Nothing is used twice, so the step is bound by memory: 28 bytes an
// element for binary32 with 32-bit moments, 16 (+ 1/16 of scales) for bfloat16 with a master copy and
// 8-bit moments.
//
// What decides a code (moments, root, scaling) is rounded operation by operation, never contracted to a fused
// multiply-add: a stochastically rounded state follows from the inputs and the seed alone, not from a compiler's choice.
//
// Decomposition: a warp takes a block of 256 elements (8 a lane: one 128-bit access of a 16-bit type,
// 256 bits of binary32, 64 bits of codes), so a block's largest magnitude is one warp reduction and no
// block is read twice.  The tensors' descriptions travel as kernel parameters, and a warp finds the
// tensor of its block by a binary search over the tensors' first blocks in constant memory.
#include <cuda_fp8.h>

#include <cmath>

#include "fewbit_device.cuh"
#include "fewbit_packed.cuh"

namespace fewbit {
bool pdl_enabled();
int device_sm_count(cudaError_t *err);

namespace {

constexpr int kBlock = FEWBIT_ADAMW_BLOCK;
// CTAs on an SM.  Measured: binary32 with 32-bit moments, 8 layers of width 640 and 1999 words (1.14 GB moved), 189 us = 6.0
// TB/s, 92 % of the copy bandwidth, where memory bounds it (3 and 5 CTAs: 195 and 202); bfloat16 with a master copy and 8-bit
// moments, 24 layers of width 1280 and 32003 words (8.24 GB), 1750 us = 4.7 TB/s, 72 %: 650 instructions for a warp's
// block keep 68 % of the issue slots busy, most of them for the codes, their noise and the roots.  Copying a warp's next block to
// shared memory meanwhile costs more instructions than the waits it saves (8 to 9 %, with 3 CTAs 2 to 3 %).
constexpr int kAdamThreads = 256, kAdamCtas = 4;

struct AdamTensor {
    void *param;
    const void *grad;
    void *m, *v;
    float *m_scale, *v_scale;
    float *master;
    unsigned long long n;        // bit 63: every buffer allows the wide accesses
};
constexpr unsigned long long kWideBit = 1ull << 63;

struct AdamScalars {
    float beta1, one_minus_beta1, beta2, one_minus_beta2;
    float keep;                  // 1 - lr * weight_decay
    float step_size;             // lr / (1 - beta1^step)
    float inv_root_bc2;          // 1 / sqrt(1 - beta2^step)
    float eps;
    uint32_t seed;
    uint32_t block0;             // blocks of the call's tensors before this launch
    const float *grad_scale;
};

// The descriptions are passed by value: a launch of a few tensors should not carry the parameters of
// hundreds (4 KB against 28 KB of parameters).
constexpr int kFewTensors = 48, kManyTensors = 400;
template <int CAP>
struct AdamBatch {
    AdamScalars s;
    uint32_t count;
    uint32_t blocks;             // of all tensors of this launch
    uint32_t first[CAP];         // first block of each tensor
    AdamTensor t[CAP];
};

// 32 random bits for a place: a Weyl step (place * kWeyl + seed, which the caller takes), then two multiply-xorshift rounds
// (odd constants from the golden ratio and the roots of 2 and 3).  The last shift is left to whoever takes the two halves.
constexpr uint32_t kWeyl = 0x9E3779B1u;
__device__ __forceinline__ uint32_t random_bits(uint32_t x) {
    x = (x ^ (x >> 15)) * 0x6A09E667u;
    return (x ^ (x >> 13)) * 0xBB67AE85u;
}

// Magnitude u in [0, 448 (1 + 2^-22)] to an e4m3 code, in the low byte, rounded up where the 20 bits cut from the mantissa
// plus `noise` (20 bits, the last 4 zero) carry.  From 2^-6 on the codes step as the mantissa does; below it they have the
// fixed step 2^-9, which u / 2 + 2^-7 turns into the mantissa's, and the larger of the two is the one that counts.
// ((127 - 7) * 8 = 960; code 8 is 2^-6.)
__device__ __forceinline__ uint32_t encode(float u, uint32_t noise) {
    const float t = fmaxf(u, fmaf(u, 0.5f, 0.0078125f));
    return (__float_as_uint(t) + noise - (960u << 20)) >> 20;
}
__device__ __forceinline__ uint32_t low_bytes(uint32_t a, uint32_t b, uint32_t c, uint32_t d) {
    return __byte_perm(__byte_perm(a, b, 0x0040), __byte_perm(c, d, 0x0040), 0x5410);
}
__device__ __forceinline__ uint32_t high_bytes(uint32_t a, uint32_t b, uint32_t c, uint32_t d) {
    return __byte_perm(__byte_perm(a, b, 0x0073), __byte_perm(c, d, 0x0073), 0x5410);
}
__device__ __forceinline__ float max_nan(float a, float b) {          // NaN if one of them is
    float d;
    asm("max.NaN.f32 %0, %1, %2;" : "=f"(d) : "f"(a), "f"(b));
    return d;
}

__device__ __forceinline__ void decode4(uint32_t w, float scale, float *out) {
    const __half2_raw lo = __nv_cvt_fp8x2_to_halfraw2(static_cast<__nv_fp8x2_storage_t>(w & 0xffffu), __NV_E4M3);
    const __half2_raw hi = __nv_cvt_fp8x2_to_halfraw2(static_cast<__nv_fp8x2_storage_t>(w >> 16), __NV_E4M3);
    const float2 a = __half22float2(__half2(lo)), b = __half22float2(__half2(hi));
    mul2(out[0], out[1], a.x, a.y, scale, scale);
    mul2(out[2], out[3], b.x, b.y, scale, scale);
}

// (scale to store, factor from value times `lift` to code) of a block whose largest magnitude has the bits `top`.
__device__ __forceinline__ void block_scale(uint32_t top, float lift, float &scale, float &factor) {
    const float t = __uint_as_float(top);
    if (top >= 0x7f800000u) { scale = __uint_as_float(0x7fc00000u); factor = 0.0f; }   // inf or NaN in the block
    else if (top < 0x00800000u) { scale = 0.0f; factor = 0.0f; }                        // the scale would have few bits or none
    else { scale = t * (1.0f / 448.0f); factor = __fmul_rn(__frcp_rn(__fmul_rn(t, lift)), 448.0f); }
}

template <typename T>
__device__ __forceinline__ void load8_some(const T *p, float (&v)[8], int valid, bool wide) {
    if (wide) { load8(p, v, true); return; }
#pragma unroll
    for (int e = 0; e < 8; ++e) v[e] = e < valid ? load1(p + e) : 0.0f;
}
template <typename T>
__device__ __forceinline__ void store8_some(T *p, const float (&v)[8], int valid, bool wide) {
    if (wide) { store8(p, v, true); return; }
#pragma unroll
    for (int e = 0; e < 8; ++e)
        if (e < valid) store1(p + e, v[e]);
}
__device__ __forceinline__ uint2 load_codes(const uint8_t *p, int valid, bool wide) {
    uint2 w = {0u, 0u};
    if (wide) {
        asm volatile("ld.global.L1::no_allocate.v2.u32 {%0,%1}, [%2];" : "=r"(w.x), "=r"(w.y) : "l"(p) : "memory");
        return w;
    }
#pragma unroll
    for (int e = 0; e < 8; ++e)
        if (e < valid) (e < 4 ? w.x : w.y) |= static_cast<uint32_t>(p[e]) << (8 * (e & 3));
    return w;
}
__device__ __forceinline__ void store_codes(uint8_t *p, uint2 w, int valid, bool wide) {
    if (wide) { asm volatile("st.global.v2.u32 [%0], {%1,%2};" :: "l"(p), "r"(w.x), "r"(w.y) : "memory"); return; }
#pragma unroll
    for (int e = 0; e < 8; ++e)
        if (e < valid) p[e] = static_cast<uint8_t>((e < 4 ? w.x : w.y) >> (8 * (e & 3)));
}

// One block: what a warp does with 8 elements of each lane, `valid` of them there.  WIDE: all of them, on aligned buffers.
template <typename T, bool EIGHT, bool MASTER, bool WIDE>
__device__ __forceinline__ void update_block(const AdamTensor &t, const AdamScalars &s, float gs, uint32_t b, uint32_t block, size_t at, int valid) {
    constexpr bool wide = WIDE;
    const int lane = threadIdx.x & 31;
    float p[8], g[8], m[8], v[8], r[8];
    load8_some(static_cast<const T *>(t.grad) + at, g, valid, wide);
    if constexpr (MASTER) load8_some(t.master + at, p, valid, wide);
    else load8_some(static_cast<const T *>(t.param) + at, p, valid, wide);
    if constexpr (EIGHT) {
        const uint2 cm = load_codes(static_cast<const uint8_t *>(t.m) + at, valid, wide);
        const uint2 cv = load_codes(static_cast<const uint8_t *>(t.v) + at, valid, wide);
        const float sm = t.m_scale[block], sv = t.v_scale[block];
        decode4(cm.x, sm, m); decode4(cm.y, sm, m + 4);
        decode4(cv.x, sv, v); decode4(cv.y, sv, v + 4);
#pragma unroll
        for (int e = 0; e < 8; e += 2) mul2(v[e], v[e + 1], v[e], v[e + 1], v[e], v[e + 1]);
    } else {
        load8_some(static_cast<const float *>(t.m) + at, m, valid, wide);
        load8_some(static_cast<const float *>(t.v) + at, v, valid, wide);
    }
    if constexpr (!WIDE) {                                         // places past the tensor's end are zeros, whatever the block's scale
#pragma unroll
        for (int e = 0; e < 8; ++e)
            if (e >= valid) m[e] = v[e] = 0.0f;
    }
    float top_m = 0.0f, top_r = 0.0f;
#pragma unroll
    for (int e = 0; e < 8; e += 2) {
        // Packed products, but scalar sums: the compiler fuses a packed product with a packed sum.
        float x0, x1, y0, y1;
        mul2(g[e], g[e + 1], g[e], g[e + 1], gs, gs);
        mul2(x0, x1, m[e], m[e + 1], s.beta1, s.beta1);
        mul2(y0, y1, g[e], g[e + 1], s.one_minus_beta1, s.one_minus_beta1);
        m[e] = __fadd_rn(x0, y0);
        m[e + 1] = __fadd_rn(x1, y1);
        mul2(x0, x1, v[e], v[e + 1], s.beta2, s.beta2);
        mul2(y0, y1, g[e], g[e + 1], g[e], g[e + 1]);
        mul2(y0, y1, y0, y1, s.one_minus_beta2, s.one_minus_beta2);
        v[e] = __fadd_rn(x0, y0);
        v[e + 1] = __fadd_rn(x1, y1);
    }
#pragma unroll
    for (int e = 0; e < 8; ++e) {
        r[e] = __fsqrt_rn(v[e]);                                  // (correctly rounded: codes must not depend on how it is computed)
        // (two ulp of the update: far below the parameter's own rounding)
        p[e] = fmaf(p[e], s.keep, -s.step_size * __fdividef(m[e], fmaf(r[e], s.inv_root_bc2, s.eps)));
        if constexpr (EIGHT) {
            top_m = max_nan(top_m, fabsf(m[e]));
            top_r = max_nan(top_r, r[e]);
        }
    }
    if constexpr (MASTER) store8_some(t.master + at, p, valid, wide);
    store8_some(static_cast<T *>(t.param) + at, p, valid, wide);
    if constexpr (EIGHT) {
        float scale_m, factor_m, scale_r, factor_r;
        // 448 / t overflows for t up to 448 / 2^128 = 1.3e-36: first moments of that size are lifted before they are scaled (from here on
        // only their codes and signs count).  Roots are 2^-74.5 at least, or zero.
        const uint32_t most_m = __reduce_max_sync(0xffffffffu, __float_as_uint(top_m));
        const bool low = most_m < 0x0d800000u;                    // 2^-100
        if (low) {
#pragma unroll
            for (int e = 0; e < 8; ++e) m[e] = __fmul_rn(m[e], 0x1p64f);
        }
        block_scale(most_m, low ? 0x1p64f : 1.0f, scale_m, factor_m);
        block_scale(__reduce_max_sync(0xffffffffu, __float_as_uint(top_r)), 1.0f, scale_r, factor_r);
        uint32_t cm[8], cr[8], wm[2], wr[2];
        const uint32_t place = ((s.block0 + b) * kBlock + lane * 8) * kWeyl + s.seed;
#pragma unroll
        for (int e = 0; e < 8; e += 2) {
            float um[2], ur[2];
            mul2(um[0], um[1], fabsf(m[e]), fabsf(m[e + 1]), factor_m, factor_m);
            mul2(ur[0], ur[1], r[e], r[e + 1], factor_r, factor_r);
#pragma unroll
            for (int x = 0; x < 2; ++x) {
                const uint32_t h = random_bits(place + (e + x) * kWeyl);
                cm[e + x] = encode(um[x], ((h << 4) ^ (h >> 12)) & 0xffff0u);
                cr[e + x] = encode(ur[x], (h >> 12) & 0xffff0u);
            }
        }
#pragma unroll
        for (int k = 0; k < 2; ++k) {
            wm[k] = low_bytes(cm[4 * k], cm[4 * k + 1], cm[4 * k + 2], cm[4 * k + 3]);
            wm[k] |= high_bytes(__float_as_uint(m[4 * k]), __float_as_uint(m[4 * k + 1]), __float_as_uint(m[4 * k + 2]), __float_as_uint(m[4 * k + 3])) & 0x80808080u;
            wr[k] = low_bytes(cr[4 * k], cr[4 * k + 1], cr[4 * k + 2], cr[4 * k + 3]);
            if ((wr[k] - 0x01010101u) & ~wr[k] & 0x80808080u) {   // some code is 0 (rare): only that of a zero may be
#pragma unroll
                for (int e = 0; e < 4; ++e)
                    if (((wr[k] >> (8 * e)) & 0xffu) == 0 && __fmul_rn(r[4 * k + e], factor_r) > 0.0f) wr[k] |= 1u << (8 * e);
            }
        }
        store_codes(static_cast<uint8_t *>(t.m) + at, make_uint2(wm[0], wm[1]), valid, wide);
        store_codes(static_cast<uint8_t *>(t.v) + at, make_uint2(wr[0], wr[1]), valid, wide);
        if (lane == 0) { t.m_scale[block] = scale_m; t.v_scale[block] = scale_r; }
    } else {
        store8_some(static_cast<float *>(t.m) + at, m, valid, wide);
        store8_some(static_cast<float *>(t.v) + at, v, valid, wide);
    }
}

template <typename T, bool EIGHT, bool MASTER, int CAP>
__global__ void __launch_bounds__(kAdamThreads, kAdamCtas)
adamw_kernel(const __grid_constant__ AdamBatch<CAP> a) {
    pdl_launch_dependents();
    const int lane = threadIdx.x & 31;
    const uint32_t warps = gridDim.x * (kAdamThreads / 32);
    pdl_wait();
    const float gs = a.s.grad_scale ? *a.s.grad_scale : 1.0f;
    uint32_t lo = 0;
    for (uint32_t b = blockIdx.x * (kAdamThreads / 32) + (threadIdx.x >> 5); b < a.blocks; b += warps) {
        if (lo + 1 < a.count && a.first[lo + 1] <= b) {      // not the last block's tensor: the last one that starts at or before b
            uint32_t hi = a.count;
            while (hi - lo > 1) {
                const uint32_t mid = (lo + hi) >> 1;
                if (a.first[mid] <= b) lo = mid; else hi = mid;
            }
        }
        const AdamTensor &t = a.t[lo];
        const unsigned long long n = t.n & ~kWideBit;
        const uint32_t block = b - a.first[lo];
        const size_t at = static_cast<size_t>(block) * kBlock + lane * 8;
        const int valid = at >= n ? 0 : (n - at < 8 ? static_cast<int>(n - at) : 8);
        const bool wide = (t.n & kWideBit) && static_cast<size_t>(block + 1) * kBlock <= n;   // the same for the whole warp
        if (wide) update_block<T, EIGHT, MASTER, true>(t, a.s, gs, b, block, at, valid);
        else update_block<T, EIGHT, MASTER, false>(t, a.s, gs, b, block, at, valid);
    }
}

template <typename T, bool EIGHT, bool MASTER, int CAP>
cudaError_t launch_adamw(const fewbit_adamw_tensor *tensors, const void *const *grads, int count, const AdamScalars &s,
                         int sms, cudaStream_t st) {
    static_assert(sizeof(AdamBatch<CAP>) <= 32000, "kernel parameters");
    AdamBatch<CAP> a;
    a.s = s;
    a.count = static_cast<uint32_t>(count);
    uint32_t at = 0;
    for (int i = 0; i < count; ++i) {
        const fewbit_adamw_tensor &t = tensors[i];
        const uintptr_t value = reinterpret_cast<uintptr_t>(t.param) | reinterpret_cast<uintptr_t>(grads[i]);
        const uintptr_t moment = reinterpret_cast<uintptr_t>(t.exp_avg) | reinterpret_cast<uintptr_t>(t.exp_avg_sq);
        const bool wide = (value & (8 * sizeof(T) - 1)) == 0 && (moment & (EIGHT ? 7 : 31)) == 0 &&
                          (reinterpret_cast<uintptr_t>(t.master) & 31) == 0;
        a.first[i] = at;
        a.t[i] = {t.param, grads[i], t.exp_avg, t.exp_avg_sq, t.exp_avg_scale, t.exp_avg_sq_scale, t.master,
                  t.n | (wide ? kWideBit : 0)};
        at += static_cast<uint32_t>((t.n + kBlock - 1) / kBlock);
    }
    a.blocks = at;
    const unsigned want = (at + kAdamThreads / 32 - 1) / (kAdamThreads / 32);
    const unsigned most = static_cast<unsigned>(sms) * kAdamCtas;
    return launch_pdl(adamw_kernel<T, EIGHT, MASTER, CAP>, want < most ? want : most, kAdamThreads, 0, st, pdl_enabled(), a);
}

template <typename T, bool EIGHT, bool MASTER>
cudaError_t launch_adamw_sized(const fewbit_adamw_tensor *tensors, const void *const *grads, int count, const AdamScalars &s,
                               int sms, cudaStream_t st) {
    return count <= kFewTensors ? launch_adamw<T, EIGHT, MASTER, kFewTensors>(tensors, grads, count, s, sms, st)
                                : launch_adamw<T, EIGHT, MASTER, kManyTensors>(tensors, grads, count, s, sms, st);
}

using AdamLaunch = cudaError_t (*)(const fewbit_adamw_tensor *, const void *const *, int, const AdamScalars &, int, cudaStream_t);
const AdamLaunch kAdam[3][2][2] = {      // [dtype][8-bit moments][master copy]
    {{launch_adamw_sized<float, false, false>, nullptr}, {launch_adamw_sized<float, true, false>, nullptr}},
    {{launch_adamw_sized<__nv_bfloat16, false, false>, launch_adamw_sized<__nv_bfloat16, false, true>},
     {launch_adamw_sized<__nv_bfloat16, true, false>, launch_adamw_sized<__nv_bfloat16, true, true>}},
    {{launch_adamw_sized<__half, false, false>, launch_adamw_sized<__half, false, true>},
     {launch_adamw_sized<__half, true, false>, launch_adamw_sized<__half, true, true>}},
};

inline bool misaligned(const void *p, uintptr_t a) { return (reinterpret_cast<uintptr_t>(p) & (a - 1)) != 0; }

}  // namespace
}  // namespace fewbit

extern "C" fewbit_status fewbit_adamw_step(const fewbit_adamw_tensor *tensors, const void *const *grads, int count,
                                           const fewbit_adamw_options *o, void *stream) {
    using namespace fewbit;
    if (o == nullptr || count < 0 || !valid_dtype(o->dtype) || (o->state_bits != 8 && o->state_bits != 32)) return FEWBIT_ERR_INVALID_ARG;
    if (o->step < 1 || !(o->beta1 >= 0 && o->beta1 < 1) || !(o->beta2 >= 0 && o->beta2 < 1) || !(o->eps >= 0) || !std::isfinite(o->eps) ||
        !(o->lr >= 0) || !std::isfinite(o->lr) || !(o->weight_decay >= 0) || !std::isfinite(o->weight_decay) ||
        misaligned(o->grad_scale_device, 4))
        return FEWBIT_ERR_INVALID_ARG;
    if (count == 0) return FEWBIT_OK;
    if (tensors == nullptr || grads == nullptr) return FEWBIT_ERR_INVALID_ARG;
    const bool eight = o->state_bits == 8;
    const uintptr_t elem = o->dtype == FEWBIT_F32 ? 4 : 2;
    int with_master = 0, used = 0;
    for (int i = 0; i < count; ++i) {
        const fewbit_adamw_tensor &t = tensors[i];
        if (t.n == 0) continue;
        ++used;
        if (t.param == nullptr || grads[i] == nullptr || t.exp_avg == nullptr || t.exp_avg_sq == nullptr ||
            (eight && (t.exp_avg_scale == nullptr || t.exp_avg_sq_scale == nullptr)))
            return FEWBIT_ERR_INVALID_ARG;
        if (t.n > (1ull << 38)) return FEWBIT_ERR_TOO_LARGE;             // blocks are counted in 32 bits
        if (misaligned(t.param, elem) || misaligned(grads[i], elem) || misaligned(t.master, 4) ||
            (!eight && (misaligned(t.exp_avg, 4) || misaligned(t.exp_avg_sq, 4))) ||
            (eight && (misaligned(t.exp_avg_scale, 4) || misaligned(t.exp_avg_sq_scale, 4))))
            return FEWBIT_ERR_ALIGNMENT;
        with_master += t.master != nullptr;
    }
    if (used == 0) return FEWBIT_OK;
    if ((with_master != 0 && with_master != used) || (with_master && o->dtype == FEWBIT_F32)) return FEWBIT_ERR_INVALID_ARG;
    AdamScalars s;
    const double bc1 = 1.0 - std::pow(o->beta1, static_cast<double>(o->step)), bc2 = 1.0 - std::pow(o->beta2, static_cast<double>(o->step));
    s.beta1 = static_cast<float>(o->beta1);
    s.one_minus_beta1 = static_cast<float>(1.0 - o->beta1);
    s.beta2 = static_cast<float>(o->beta2);
    s.one_minus_beta2 = static_cast<float>(1.0 - o->beta2);
    s.keep = static_cast<float>(1.0 - o->lr * o->weight_decay);
    s.step_size = static_cast<float>(o->lr / bc1);
    s.inv_root_bc2 = static_cast<float>(1.0 / std::sqrt(bc2));
    s.eps = static_cast<float>(o->eps);
    s.seed = o->seed;
    s.block0 = 0;
    s.grad_scale = o->grad_scale_device;
    cudaError_t err = cudaSuccess;
    const int sms = device_sm_count(&err);
    for (int at = 0; err == cudaSuccess && at < count;) {
        int n = 0;
        unsigned long long blocks = 0;
        while (at + n < count && n < kManyTensors) {
            const unsigned long long more = (tensors[at + n].n + kBlock - 1) / kBlock;
            if (n > 0 && blocks + more > 0xfff00000ull) break;
            blocks += more;
            ++n;
        }
        if (blocks > 0) {
            err = kAdam[o->dtype][eight][with_master != 0](tensors + at, grads + at, n, s, sms, static_cast<cudaStream_t>(stream));
            if (err == cudaSuccess) g_launches.fetch_add(1, std::memory_order_relaxed);
        }
        s.block0 += static_cast<uint32_t>(blocks);
        at += n;
    }
    if (err != cudaSuccess) { t_last_cuda_error = static_cast<int>(err); return FEWBIT_ERR_CUDA; }
    return FEWBIT_OK;
}
