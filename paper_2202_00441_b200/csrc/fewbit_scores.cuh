// What stands between attention's products and its softmax (fewbit_attention_scores): a cap, a bias by distance, masks by
// prefix and documents.  Included by the attention kernels.
//
// Mathematics, d = key - row - (k_len - q_len), s the product, c the scale, in units of ln 2:
//   z = c s log2 e,  or  cap tanh(c s / cap) log2 e;   z -= slope |d| log2 e;   z += B[clamp(d)] log2 e
// and backward, with t the tanh: dS = dZ (1 - t^2), dB[e] = sum of dZ over all pairs at distance e.
//
// tanh: an odd polynomial of the product, scale and cap folded into its coefficients: of degree 5 where no product of a warp's 32 x 32
// piece passes 0.3 caps (relative error 1.2e-6), of degree 11 up to the cap itself (6.1e-7), both found by Lawson's reweighted least
// squares; two results of the exponential unit otherwise.  FMA and exponential pipe are what bounds the capped kernels: the
// polynomials take 4 and 7 multiplications an element.  (tanh.approx.f32 has 11 bits: with a cap of 50 a score would be off by 0.02.)
// Bias: a warp works on 32 rows x 32 keys; where all of them lie further apart than the table reaches, the bias is one number,
// else each element's is read, 32 neighbouring ones at a time.
// Measured, bfloat16, 4 x 2048 rows, 16 heads on 4 of 128, causal, forward and backward, single passes: plain scores 90 and 254 us, cap 50 121 and
// 355, slopes 127 and 342, a table of 128 distances 123 and 347 (396 with its gradient).  What a tile costs more is the chain of one warp's
// instructions: the tensor cores wait for it half of the time.
// Documents: a lane holds the document of one key, and each document among a warp's 32 keys (mostly one or two) becomes one
// word of votes.  Tiles in front of the first and behind the last that shares a document with the CTA's own are skipped.
#pragma once

#include <cfloat>
#include <climits>
#include <type_traits>

#include "fewbit_tensor_core.cuh"

namespace fewbit {
namespace attn {

using namespace tc;

struct Scores {
    float cap_in, cap_out;            // scale / cap, cap * log2(e)
    float cap_out_2;                  // cap_out^-2
    float near_odd[3], odd[6];        // capped scores of products up to near_limit and odd_limit: s Q(s^2), in units of ln 2
    float near_limit, odd_limit;
    const float *slopes, *bias;
    int reach;                        // the table's largest distance
    const int *prefix, *q_docs, *k_docs;
    // the bias's gradient: sums by distance of each key tile's near row tiles, sums of the far ones, what was written
    float *near, *far;
    float *far_delta;                 // -delta of each row (128 for a row tile) whose place in the statistics something else takes
    int4 *written;                    // row tiles [x, y), k_len - q_len, number of the key tile + 1 (0: none has this place)
    int places;                       // for key tiles, of a sequence and head, or of all packed sequences for a head
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

// -slope * log2(e), finite (a level key's distance of 0 is multiplied by it).
__device__ __forceinline__ float slope_of(float slope) {
    const float m = -slope * 1.4426950408889634f;
    return m < -FLT_MAX ? -FLT_MAX : m;
}

// Any a, relative error below 2^-19: 1 - 2 / (1 + e^2a) is off by 2^-21 at most, which small values do not bear (a cap far above
// the scores multiplies it).
__device__ __forceinline__ float tanh_any(float a) {
    float r;
    asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(1.0f + exp2_fast(2.885390081777927f * a)));
    const float y = a * a, near = a * fmaf(y, fmaf(y, 0.12633946537971497f, -0.33310022950172424f), 0.9999988675117493f);
    return fabsf(a) < 0.3f ? near : fmaf(-2.0f, r, 1.0f);
}
// One product's capped score.
__device__ __forceinline__ float bend_one(const Scores &sc, float s) { return tanh_any(s * sc.cap_in) * sc.cap_out; }
__device__ __forceinline__ float abs_max3(float a, float b, float c) {
    float d;
    asm("max.f32 %0, %1, %2, %3;" : "=f"(d) : "f"(a), "f"(fabsf(b)), "f"(fabsf(c)));
    return d;
}
__device__ __forceinline__ float largest(const uint32_t (&s)[32]) {   // magnitude
    float high[2] = {0.0f, 0.0f};
#pragma unroll
    for (int e = 0; e < 32; e += 2) high[e / 2 % 2] = abs_max3(high[e / 2 % 2], __uint_as_float(s[e]), __uint_as_float(s[e + 1]));
    return fmaxf(high[0], high[1]);
}
// 32 products to capped scores plus `add`, with the shortest form that the warp's largest product (`high`) allows.  Returns whether
// one of the warp's may lie past the cap.
template <int MODE, bool ADD>
__device__ __forceinline__ bool bend(const Scores &sc, float high, uint32_t (&s)[32], float add) {
    auto odd = [&](auto degree, const float *c) {                     // s Q(s^2)
        constexpr int N = decltype(degree)::value;
#pragma unroll
        for (int e = 0; e < 32; e += 2) {
            const float a = __uint_as_float(s[e]), b = __uint_as_float(s[e + 1]);
            float y0, y1, q0, q1;
            mul2(y0, y1, a, b, a, b);
            fma2(q0, q1, y0, y1, c[N], c[N], c[N - 1], c[N - 1]);
#pragma unroll
            for (int k = N - 2; k >= 0; --k) fma2(q0, q1, q0, q1, y0, y1, c[k], c[k]);
            if (ADD) fma2(q0, q1, q0, q1, a, b, add, add);
            else mul2(q0, q1, q0, q1, a, b);
            s[e] = __float_as_uint(q0);
            s[e + 1] = __float_as_uint(q1);
        }
    };
    if (MODE == 1 && !__any_sync(0xffffffffu, high > sc.near_limit)) {   // (with biases, a rare pair, the code's size counts for more)
        odd(std::integral_constant<int, 2>{}, sc.near_odd);
        return false;
    } else if (!__any_sync(0xffffffffu, high > sc.odd_limit)) {
        odd(std::integral_constant<int, 5>{}, sc.odd);
        return false;
    } else {
#pragma unroll
        for (int e = 0; e < 32; ++e) {
            const float t = tanh_any(__uint_as_float(s[e]) * sc.cap_in);
            s[e] = __float_as_uint(ADD ? fmaf(t, sc.cap_out, add) : t * sc.cap_out);
        }
        return true;
    }
}
// 1 - t^2 of 32 capped scores in 16 bits each, for half the registers.  As binary16 it is off by up to 2^-11, an eighth of what dS
// loses when it is rounded to bfloat16, but as much as dS loses as binary16.  There (FINE) it is kept, up to the cap, where 1 - t^2 is
// above 0.4, in steps of 2^-15, off by 2^-16; past the cap (`steep`) with 3 bits for the exponent and 13 for the mantissa, off by
// 2^-14 of it or 2^-20, less than t itself is.  Errors of dQ and dK against that of rounding the results alone, 1000 rows and keys:
// 1.6 and 1.4 (a cap of 20), as without a cap, instead of 1.8 and 1.6; 1.4 and 1.4 (5) instead of 1.7 and 1.7.
template <bool FINE>
__device__ __forceinline__ void bent_slopes(float cap_out_2, bool steep, const uint32_t (&z)[32], uint32_t (&bent)[16]) {
    auto slopes = [&](float one, auto pack) {
#pragma unroll
        for (int e = 0; e < 16; ++e) {
            float a, b;
            mul2(a, b, __uint_as_float(z[2 * e]), __uint_as_float(z[2 * e + 1]), __uint_as_float(z[2 * e]), __uint_as_float(z[2 * e + 1]));
            fma2(a, b, a, b, -cap_out_2, -cap_out_2, one, one);
            bent[e] = pack(a, b);
        }
    };
    if (!FINE) {
        slopes(1.0f, [](float a, float b) { return pack2<__half>(a, b); });
    } else if (!steep) {                                              // (above 256 a number's last 16 bits count 2^-15)
        slopes(257.0f, [](float a, float b) { return __byte_perm(__float_as_uint(a), __float_as_uint(b), 0x5410); });
    } else {                                                          // (1 is 7 << 23 after the product)
        slopes(1.0f, [](float a, float b) {
            mul2(a, b, a, b, 0x1p-120f, 0x1p-120f);
            return __byte_perm((__float_as_uint(a) + 0x200u) >> 10, (__float_as_uint(b) + 0x200u) >> 10, 0x5410);
        });
    }
}
// 32 values times them
template <bool FINE>
__device__ __forceinline__ void times_bent(const uint32_t (&bent)[16], bool steep, float (&x)[32]) {
    auto times = [&](auto unpack) {
#pragma unroll
        for (int c = 0; c < 16; ++c) {
            float a, b;
            unpack(bent[c], a, b);
            mul2(x[2 * c], x[2 * c + 1], x[2 * c], x[2 * c + 1], a, b);
        }
    };
    if (!FINE) {
        times([](uint32_t w, float &a, float &b) {
            const float2 f = __half22float2(*reinterpret_cast<const __half2 *>(&w));
            a = f.x;
            b = f.y;
        });
    } else if (!steep) {
        times([](uint32_t w, float &a, float &b) {
            add2(a, b, __uint_as_float(__byte_perm(w, 0x43800000u, 0x7610)), __uint_as_float(__byte_perm(w, 0x43800000u, 0x7632)), -256.0f, -256.0f);
        });
    } else {
        times([](uint32_t w, float &a, float &b) {
            mul2(a, b, __uint_as_float((w & 0xffffu) << 10), __uint_as_float(w >> 16 << 10), 0x1p120f, 0x1p120f);
        });
    }
}

// Whether rows and keys of a warp's 32 x 32 piece (`least`: the distance of its last row and first key; the others are up to 62
// more) are all further apart than the table reaches: -1 the keys lie behind, 1 ahead, 0 not all.
__device__ __forceinline__ int beyond(int least, int reach) { return least + 62 <= -reach ? -1 : least >= reach ? 1 : 0; }

// The bias of 32 products or capped scores (factor: what brings them to units of ln 2), value x at distance away + at(x) of a
// warp's 32 x 32 piece whose smallest distance is `least`.  Returns whether every result is finite where the scores are (tables
// may hold -inf).  look(x): the table's value for it in units of ln 2, for pieces within the table's reach.
template <typename At, typename Look>
__device__ __forceinline__ bool add_bias(const Scores &sc, const Mods &m, float factor, int away, int least, uint32_t (&s)[32], At at, Look look) {
    if (sc.slopes != nullptr) {
        const float first = static_cast<float>(away);
#pragma unroll
        for (int x = 0; x < 32; x += 2) {                             // (one pass for both takes 5 % longer)
            float v0, v1;
            mul2(v0, v1, __uint_as_float(s[x]), __uint_as_float(s[x + 1]), factor, factor);
            s[x] = __float_as_uint(v0);
            s[x + 1] = __float_as_uint(v1);
        }
        if (m.slope != 0.0f) {
#pragma unroll
            for (int x = 0; x < 32; ++x) s[x] = __float_as_uint(fmaf(m.slope, fabsf(first + static_cast<float>(at(x))), __uint_as_float(s[x])));
        }
        factor = 1.0f;
    }
    const bool finite = m.slope > -1e29f;                             // (distances are below 2^31: no product with such a slope overflows)
    if (m.bias == nullptr) return finite;
    const int far = beyond(least, sc.reach);
    if (far != 0) {
        const float b = __ldg(m.bias + (far < 0 ? -sc.reach : sc.reach)) * 1.4426950408889634f;
#pragma unroll
        for (int x = 0; x < 32; x += 2) {
            float v0, v1;
            fma2(v0, v1, __uint_as_float(s[x]), __uint_as_float(s[x + 1]), factor, factor, b, b);
            s[x] = __float_as_uint(v0);
            s[x + 1] = __float_as_uint(v1);
        }
        return finite && b > -INFINITY;
    }
#pragma unroll
    for (int x = 0; x < 32; ++x) s[x] = __float_as_uint(fmaf(__uint_as_float(s[x]), factor, look(x)));
    return false;
}

// The score of one product at distance `away`, with the roundings of the forms above.
__device__ __forceinline__ float shape_one(const Scores &sc, const Mods &m, float scale_log2, int away, float s) {
    if (sc.capped) {
        s = bend_one(sc, s);
        scale_log2 = 1.0f;
    }
    if (sc.slopes != nullptr) {
        s *= scale_log2;
        if (m.slope != 0.0f) s = fmaf(m.slope, fabsf(static_cast<float>(away)), s);
        scale_log2 = 1.0f;
    }
    return m.bias == nullptr ? s : fmaf(s, scale_log2, __ldg(m.bias + max(-sc.reach, min(sc.reach, away))) * 1.4426950408889634f);
}

// A thread's row and 32 neighbouring keys from `away` on (the distance of the first; lanes' rows are neighbours: away falls by
// one with each lane).  s: products in, scores in units of ln 2 out (MODE 1: only with a cap).  GRADIENT: bent gets 1 - t^2 of each pair
// (steep: in which form, see bent_slopes).
template <int MODE, bool GRADIENT, bool FINE>
__device__ __forceinline__ bool shape_scores(const Scores &sc, const Mods &m, float scale_log2, int away, uint32_t (&s)[32], uint32_t (&bent)[16], bool &steep) {
    float factor = scale_log2;
    if (sc.capped) {
        steep = bend<MODE, false>(sc, largest(s), s, 0.0f);
        factor = 1.0f;
        if constexpr (GRADIENT) bent_slopes<FINE>(sc.cap_out_2, steep, s, bent);
    }
    if constexpr (MODE == 1) return true;
    return add_bias(sc, m, factor, away, uniform(away) - 31, s, [](int x) { return x; },
                    [&](int x) { return __ldg(m.bias + max(-sc.reach, min(sc.reach, away + x))) * 1.4426950408889634f; });
}
// The same for the transposed scores of the dK and dV kernel: s[16 (k / 2) + 4 c + 2 (k % 2) + e] is of key 8 k and row 8 c + e
// from this thread's first ones on, which are `away` apart.
template <int MODE, bool FINE>
__device__ __forceinline__ void shape_transposed(const Scores &sc, const Mods &m, float scale_log2, int away, int least, uint32_t (&s)[32], uint32_t (&bent)[16],
                                                 bool &steep) {
    float factor = scale_log2;
    if (sc.capped) {
        steep = bend<MODE, false>(sc, largest(s), s, 0.0f);
        factor = 1.0f;
        bent_slopes<FINE>(sc.cap_out_2, steep, s, bent);
    }
    if constexpr (MODE == 1) return;
    // key minus row takes 14 values: 8 (k - c) - e
    float b[14];
    if (m.bias != nullptr && beyond(least, sc.reach) == 0) {
#pragma unroll
        for (int y = 0; y < 14; ++y) b[y] = __ldg(m.bias + max(-sc.reach, min(sc.reach, away + 8 * (y / 2 - 3) - y % 2))) * 1.4426950408889634f;
    }
    add_bias(sc, m, factor, away, least, s, [](int x) { return 8 * (2 * (x / 16) + x / 2 % 2) - 8 * (x / 4 % 4) - x % 2; },
                    [&](int x) { return b[2 * (2 * (x / 16) + x / 2 % 2 - x / 4 % 4 + 3) + x % 2]; });
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

// Tiles [lo, hi) of `n` tiles (documents `theirs`, `their_len` of them) in which a document of `mine` [mine_first, mine_end), at
// most 32 * ROWS of them, may be: their smallest and largest documents overlap.  In two parts, with a barrier of the whole CTA
// between them: scan_tiles lets every warp look at every 20th tile, eight of them waiting for memory together, and leaves what it
// found in its place of shared memory; scanned_tiles puts that together.
constexpr int kScanWarps = 20;
template <int ROWS>
__device__ __forceinline__ void scan_tiles(const int *mine, int mine_first, int mine_end, const int *theirs, int their_len, int n, int2 *place) {
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    constexpr int kTogether = 8;
    int smallest = INT_MAX, greatest = INT_MIN, lo = INT_MAX, hi = 0;
    if (n > warp) {
#pragma unroll
        for (int i = 0; i < ROWS; ++i) {
            const int d = __ldg(mine + min(mine_first + 32 * i + lane, mine_end - 1));
            smallest = min(smallest, d);
            greatest = max(greatest, d);
        }
    }
    for (int t0 = warp; t0 < n; t0 += kTogether * kScanWarps) {
        int low[kTogether], high[kTogether];
#pragma unroll
        for (int i = 0; i < kTogether; ++i) {
            int d[4];
#pragma unroll
            for (int k = 0; k < 4; ++k) d[k] = __ldg(theirs + min((t0 + i * kScanWarps) * 128 + 32 * k + lane, their_len - 1));   // (the last one again past the end)
            low[i] = min(min(d[0], d[1]), min(d[2], d[3]));
            high[i] = max(max(d[0], d[1]), max(d[2], d[3]));
        }
        if (t0 == warp) {
            smallest = __reduce_min_sync(0xffffffffu, smallest);
            greatest = __reduce_max_sync(0xffffffffu, greatest);
        }
#pragma unroll
        for (int i = 0; i < kTogether; ++i) {
            const int t = t0 + i * kScanWarps, a = __reduce_min_sync(0xffffffffu, low[i]), b = __reduce_max_sync(0xffffffffu, high[i]);
            if (t < n && a <= greatest && b >= smallest) {
                lo = min(lo, t);
                hi = t + 1;
            }
        }
    }
    if (lane == 0) place[warp] = make_int2(lo, hi);
}
__device__ __forceinline__ int2 scanned_tiles(const int2 *place) {
    const int lane = threadIdx.x & 31;
    const int2 found = lane < kScanWarps ? place[lane] : make_int2(INT_MAX, 0);
    const int lo = __reduce_min_sync(0xffffffffu, found.x), hi = __reduce_max_sync(0xffffffffu, found.y);
    return hi == 0 ? make_int2(0, 0) : make_int2(lo, hi);
}

}  // namespace attn
}  // namespace fewbit
