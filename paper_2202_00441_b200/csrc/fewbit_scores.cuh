// What stands between attention's products and its softmax (fewbit_attention_scores): a cap, a bias by distance, masks by
// prefix and documents.  Included by the attention kernels.
//
// Mathematics, d = key - row - (k_len - q_len), s the product, c the scale, in units of ln 2:
//   z = c s log2 e,  or  cap tanh(c s / cap) log2 e;   z -= slope |d| log2 e;   z += B[clamp(d)] log2 e
// and backward, with t the tanh: dS = dZ (1 - t^2), dB[e] = sum of dZ over all pairs at distance e.
//
// tanh: where no product of a warp's piece passes the cap itself, an odd polynomial of degree 11 (relative error 6e-7 on [-1, 1],
// found by Lawson's reweighted least squares) on the FMA pipe, which has room; two results of the exponential unit otherwise.
// (tanh.approx.f32 has 11 bits: with a cap of 50 a score would be off by 0.02.)
// Bias: a warp works on 32 rows x 32 keys; where all of them lie further apart than the table reaches, the bias is one number,
// else each element's is read, 32 neighbouring ones at a time.
// Documents: a lane holds the document of one key, and each document among a warp's 32 keys (mostly one or two) becomes one
// word of votes.  Tiles in front of the first and behind the last that shares a document with the CTA's own are skipped.
#pragma once

#include "fewbit_tensor_core.cuh"

namespace fewbit {
namespace attn {

using namespace tc;

struct Scores {
    float cap_in, cap_out;            // scale / cap, cap * log2(e)
    const float *slopes, *bias;
    int reach;                        // the table's largest distance
    const int *prefix, *q_docs, *k_docs;
    // the bias's gradient: sums by distance of each key tile's near row tiles, sums of the far ones, what was written
    float *near, *far;
    int4 *written;                    // row tiles [x, y), k_len - q_len, 0
    int near_tiles;                   // places for near row tiles of one key tile
    bool capped;
};
constexpr int kFarFloats = 4 * 16 * 2;          // of one key tile and head: [CTA of the cluster][warp][behind, ahead]
constexpr int kNearFloats = 16 * 64;            // of one pair of tiles: [warp][distance]

// The first row tile (it may be negative) with a key of the key tile at k0 nearer than `most`.
__host__ __device__ __forceinline__ int first_near(int k0, int reach, int most) {
    const int past = k0 - 127 - reach - most;   // a row tile at i0 is near if past < i0
    return (past >= 0 ? past / 128 : -((127 - past) / 128)) + 1;
}

// What one CTA needs of it.
struct Mods {
    int prefix;                       // keys below it are seen by every row
    const int *q_docs, *k_docs;       // of the sequence's first row and key
    const float *bias;                // the head's, at distance 0
    float slope;                      // -slope * log2(e)
};

__device__ __forceinline__ float tanh_wide(float a) {                 // absolute error below 2^-21
    float r;
    asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(1.0f + exp2_fast(2.885390081777927f * a)));
    return fmaf(-2.0f, r, 1.0f);
}
// (t0, t1) = tanh(a0, a1) for magnitudes up to 1
__device__ __forceinline__ void tanh_small(float &t0, float &t1, float a0, float a1) {
    float y0, y1, p0, p1;
    mul2(y0, y1, a0, a1, a0, a1);
    fma2(p0, p1, y0, y1, -0.0030670601408928633f, -0.0030670601408928633f, 0.016743114218115807f, 0.016743114218115807f);
    fma2(p0, p1, p0, p1, y0, y1, -0.051605671644210815f, -0.051605671644210815f);
    fma2(p0, p1, p0, p1, y0, y1, 0.13281433284282684f, 0.13281433284282684f);
    fma2(p0, p1, p0, p1, y0, y1, -0.3332904279232025f, -0.3332904279232025f);
    fma2(p0, p1, p0, p1, y0, y1, 0.9999994039535522f, 0.9999994039535522f);
    mul2(t0, t1, p0, p1, a0, a1);
}
__device__ __forceinline__ float abs_max3(float a, float b, float c) {
    float d;
    asm("max.f32 %0, %1, %2, %3;" : "=f"(d) : "f"(a), "f"(fabsf(b)), "f"(fabsf(c)));
    return d;
}

// 32 products, in registers, to tanh(c s / cap), two neighbouring ones at a time.
__device__ __forceinline__ void bend(float cap_in, uint32_t (&s)[32]) {
    float high = 0.0f;
#pragma unroll
    for (int e = 0; e < 32; e += 2) {
        float a, b;
        mul2(a, b, __uint_as_float(s[e]), __uint_as_float(s[e + 1]), cap_in, cap_in);
        high = abs_max3(high, a, b);
        s[e] = __float_as_uint(a);
        s[e + 1] = __float_as_uint(b);
    }
    if (__any_sync(0xffffffffu, high > 1.0f)) {
#pragma unroll
        for (int e = 0; e < 32; ++e) s[e] = __float_as_uint(tanh_wide(__uint_as_float(s[e])));
    } else {
#pragma unroll
        for (int e = 0; e < 32; e += 2) {
            float a, b;
            tanh_small(a, b, __uint_as_float(s[e]), __uint_as_float(s[e + 1]));
            s[e] = __float_as_uint(a);
            s[e + 1] = __float_as_uint(b);
        }
    }
}
// 1 - t^2 of two, as binary16: 2^-12 of it, less than dS's own rounding, for half the registers
__device__ __forceinline__ uint32_t bent_slope(float t0, float t1) {
    float a, b;
    mul2(a, b, t0, t1, t0, t1);
    return pack2<__half>(1.0f - a, 1.0f - b);
}

// Whether rows and keys of a warp's 32 x 32 piece (`least`: the distance of its last row and first key; the others are up to 62
// more) are all further apart than the table reaches: -1 the keys lie behind, 1 ahead, 0 not all.
__device__ __forceinline__ int beyond(int least, int reach) { return least + 62 <= -reach ? -1 : least >= reach ? 1 : 0; }

// A thread's row and 32 neighbouring keys from `away` on (the distance of the first; lane's rows are neighbours: away falls by
// one with each lane).  s: products in, scores in units of ln 2 out.  GRADIENT: bent gets 1 - t^2 of each pair.  Returns
// whether every score is finite where the products are (bias tables may hold -inf).  For a whole warp.
template <bool GRADIENT>
__device__ __forceinline__ bool shape_scores(const Scores &sc, const Mods &m, float scale_log2, int away, uint32_t (&s)[32], uint32_t (&bent)[16]) {
    float factor = scale_log2;
    if (sc.capped) {
        bend(sc.cap_in, s);
        factor = sc.cap_out;
        if constexpr (GRADIENT) {
#pragma unroll
            for (int e = 0; e < 16; ++e) bent[e] = bent_slope(__uint_as_float(s[2 * e]), __uint_as_float(s[2 * e + 1]));
        }
    }
#pragma unroll
    for (int e = 0; e < 32; e += 2) {
        float a, b;
        mul2(a, b, __uint_as_float(s[e]), __uint_as_float(s[e + 1]), factor, factor);
        s[e] = __float_as_uint(a);
        s[e + 1] = __float_as_uint(b);
    }
    if (m.slope != 0.0f) {
        const float first = static_cast<float>(away);
#pragma unroll
        for (int e = 0; e < 32; ++e) s[e] = __float_as_uint(fmaf(m.slope, fabsf(first + static_cast<float>(e)), __uint_as_float(s[e])));
    }
    if (m.bias == nullptr) return true;
    const int far = beyond(uniform(away) - 31, sc.reach);
    if (far != 0) {
        const float b = __ldg(m.bias + (far < 0 ? -sc.reach : sc.reach)) * 1.4426950408889634f;
#pragma unroll
        for (int e = 0; e < 32; ++e) s[e] = __float_as_uint(__uint_as_float(s[e]) + b);
        return b > -INFINITY;
    }
#pragma unroll
    for (int e = 0; e < 32; ++e) {
        const float b = __ldg(m.bias + max(-sc.reach, min(sc.reach, away + e)));
        s[e] = __float_as_uint(fmaf(b, 1.4426950408889634f, __uint_as_float(s[e])));
    }
    return false;
}

// The same for the transposed scores of the dK and dV kernel: s[16 (k / 2) + 4 c + 2 (k % 2) + e] is of key 8 k and row 8 c + e
// from this thread's first ones on, which are `away` apart.
__device__ __forceinline__ bool shape_transposed(const Scores &sc, const Mods &m, float scale_log2, int away, int least, uint32_t (&s)[32], uint32_t (&bent)[16]) {
    float factor = scale_log2;
    if (sc.capped) {
        bend(sc.cap_in, s);
        factor = sc.cap_out;
#pragma unroll
        for (int e = 0; e < 16; ++e) bent[e] = bent_slope(__uint_as_float(s[2 * e]), __uint_as_float(s[2 * e + 1]));
    }
#pragma unroll
    for (int e = 0; e < 32; e += 2) {
        float a, b;
        mul2(a, b, __uint_as_float(s[e]), __uint_as_float(s[e + 1]), factor, factor);
        s[e] = __float_as_uint(a);
        s[e + 1] = __float_as_uint(b);
    }
    auto distance = [](int x) { return 8 * (2 * (x / 16) + x / 2 % 2) - 8 * (x / 4 % 4) - x % 2; };   // from the first one's
    if (m.slope != 0.0f) {
        const float first = static_cast<float>(away);
#pragma unroll
        for (int x = 0; x < 32; ++x) s[x] = __float_as_uint(fmaf(m.slope, fabsf(first + static_cast<float>(distance(x))), __uint_as_float(s[x])));
    }
    if (m.bias == nullptr) return true;
    const int far = beyond(least, sc.reach);
    if (far != 0) {
        const float b = __ldg(m.bias + (far < 0 ? -sc.reach : sc.reach)) * 1.4426950408889634f;
#pragma unroll
        for (int x = 0; x < 32; ++x) s[x] = __float_as_uint(__uint_as_float(s[x]) + b);
        return b > -INFINITY;
    }
    // key minus row takes 14 values: 8 (k - c) - e
    float b[14];
#pragma unroll
    for (int y = 0; y < 14; ++y) b[y] = __ldg(m.bias + max(-sc.reach, min(sc.reach, away + 8 * (y / 2 - 3) - y % 2)));
#pragma unroll
    for (int x = 0; x < 32; ++x) s[x] = __float_as_uint(fmaf(b[2 * (2 * (x / 16) + x / 2 % 2 - x / 4 % 4 + 3) + x % 2], 1.4426950408889634f, __uint_as_float(s[x])));
    return false;
}

// Sums over the diagonals of a warp's 32 keys x 32 rows.  v[m][e]: this thread's sum over its values with (key - row) / 8 = m - 3
// of its own and row parity e; its first key is lane / 4, its first row 2 (lane % 4).  out[x]: the sum over the warp at
// key - row = 16 (lane % 4) + 8 x + lane / 4 - 32.  For a whole warp.
__device__ __forceinline__ void sum_diagonals(const float (&v)[7][2], float (&out)[2]) {
    const int lane = threadIdx.x & 31, t = lane >> 2, b = lane & 3;
    // a thread's distance is 8 (m - 3) + lane / 4 - 2 b - e: lanes of one b turn by 2 b, so that lane / 4 is the distance's
    // rest by 8 (plus e); those that come round belong one m lower
    const int from = ((t + 2 * b) & 7) * 4 + b;
    const bool round = t + 2 * b >= 8;
    float q[16];                                                      // [m + 1 of -4 .. 3][e]
#pragma unroll
    for (int e = 0; e < 2; ++e) {
        float r[7];
#pragma unroll
        for (int m = 0; m < 7; ++m) r[m] = __shfl_sync(0xffffffffu, v[m][e], from);
#pragma unroll
        for (int m = 0; m < 8; ++m) q[2 * m + e] = round ? (m < 7 ? r[m] : 0.0f) : (m > 0 ? r[m - 1] : 0.0f);
    }
    // sums over the four b: each keeps a quarter of the 16
    float h[8], s[4];
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const float give = b & 2 ? q[i] : q[i + 8];
        h[i] = (b & 2 ? q[i + 8] : q[i]) + __shfl_xor_sync(0xffffffffu, give, 2);
    }
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const float give = b & 1 ? h[i] : h[i + 4];
        s[i] = (b & 1 ? h[i + 4] : h[i]) + __shfl_xor_sync(0xffffffffu, give, 1);
    }
    // s[2 x + e]: distance 8 (2 b + x - 4) + t - e.  Those of e = 1 move to the place before: the next t's, for t = 7 the next 8's
    const int next = ((t + 1) & 7) * 4 + b;
    const float n0 = __shfl_sync(0xffffffffu, s[1], next), n1 = __shfl_sync(0xffffffffu, s[3], next);
    const float n2 = __shfl_sync(0xffffffffu, s[1], (b + 1) & 3);
    out[0] = s[0] + (t < 7 ? n0 : n1);
    out[1] = s[2] + (t < 7 ? n1 : b < 3 ? n2 : 0.0f);
}

// The low `limit` bits of a word (any limit).
__device__ __forceinline__ uint32_t low_bits(int limit) { return limit >= 32 ? 0xffffffffu : limit <= 0 ? 0u : (1u << limit) - 1u; }

// A bit for each of 32 keys (`theirs`: lane's key's document) that is of this thread's document.  For a whole warp.
__device__ __forceinline__ uint32_t same_document(int mine, int theirs) {
    uint32_t left = 0xffffffffu, word = 0;
    while (left != 0) {
        const int document = __shfl_sync(0xffffffffu, theirs, __ffs(left) - 1);
        const uint32_t these = __ballot_sync(0xffffffffu, theirs == document);
        if (mine == document) word = these;
        left &= ~these;
    }
    return word;
}

// Tiles [lo, hi) of `n` tiles (documents `theirs`, `their_len` of them) in which a document of `mine` [mine_first, mine_end)
// may be: their smallest and largest documents overlap.  `place`: 4 words of shared memory, free.  For the whole CTA, with
// three barriers; the result is the same for all.
__device__ __forceinline__ int2 shared_tiles(const int *mine, int mine_first, int mine_end, const int *theirs, int their_len, int n, int *place) {
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, warps = blockDim.x >> 5;
    if (threadIdx.x == 0) {
        place[0] = INT_MAX; place[1] = INT_MIN;                       // smallest and largest of mine
        place[2] = INT_MAX; place[3] = 0;                             // lo, hi
    }
    __syncthreads();
    for (int at = mine_first + warp * 32; at < mine_end; at += warps * 32) {
        const int d = __ldg(mine + min(at + lane, mine_end - 1));
        const int low = __reduce_min_sync(0xffffffffu, d), high = __reduce_max_sync(0xffffffffu, d);
        if (lane == 0) {
            atomicMin(place, low);
            atomicMax(place + 1, high);
        }
    }
    __syncthreads();
    const int low = place[0], high = place[1];
    for (int t = warp; t < n; t += warps) {
        int a = INT_MAX, b = INT_MIN;
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            const int at = t * 128 + 32 * k + lane;
            if (at < their_len) {
                const int d = __ldg(theirs + at);
                a = min(a, d);
                b = max(b, d);
            }
        }
        a = __reduce_min_sync(0xffffffffu, a);
        b = __reduce_max_sync(0xffffffffu, b);
        if (lane == 0 && a <= high && b >= low) {
            atomicMin(place + 2, t);
            atomicMax(place + 3, t + 1);
        }
    }
    __syncthreads();
    return uniform(place[3]) == 0 ? make_int2(0, 0) : make_int2(uniform(place[2]), uniform(place[3]));
}

}  // namespace attn
}  // namespace fewbit
