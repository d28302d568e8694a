// Random words that are drawn again wherever they are needed: Philox4x32-10 (Salmon, Moraes, Dror and Shaw, Parallel
// random numbers: as easy as 1, 2, 3, 2011).  A block of four words is a function of a counter and a key: element e of a tensor
// takes word e % 4 of the block whose counter is (e / 4, its upper half, place, 0), with the seed's halves as key.
#pragma once

#include <cstdint>

namespace fewbit {

struct RandomKeys {              // of the ten rounds
    uint32_t a[10], b[10];
};

__host__ __device__ __forceinline__ RandomKeys random_keys(uint64_t seed) {
    RandomKeys k;
#pragma unroll
    for (int i = 0; i < 10; ++i) {
        k.a[i] = static_cast<uint32_t>(seed) + i * 0x9E3779B9u;
        k.b[i] = static_cast<uint32_t>(seed >> 32) + i * 0xBB67AE85u;
    }
    return k;
}

// The words of elements [4 group, 4 group + 4), group = high 2^32 + low.  Where `high` is the same for several groups, half of
// the first two rounds' products are too, and the compiler takes them once.
__device__ __forceinline__ uint4 random_words(const RandomKeys &k, uint32_t low, uint32_t high, uint32_t place) {
    uint32_t c0 = low, c1 = high, c2 = place, c3 = 0;
#pragma unroll
    for (int i = 0; i < 10; ++i) {
        const uint64_t m0 = static_cast<uint64_t>(c0) * 0xD2511F53u, m1 = static_cast<uint64_t>(c2) * 0xCD9E8D57u;
        c0 = static_cast<uint32_t>(m1 >> 32) ^ c1 ^ k.a[i];
        c1 = static_cast<uint32_t>(m1);
        c2 = static_cast<uint32_t>(m0 >> 32) ^ c3 ^ k.b[i];
        c3 = static_cast<uint32_t>(m0);
    }
    return make_uint4(c0, c1, c2, c3);
}

// What dropout needs to know: an element is kept where its word is at least `limit`.
struct Drop {
    RandomKeys keys;             // of a seed that the host knows: operands straight from the kernel's parameters
    uint64_t seed;
    const int64_t *seed_device;  // added to it, if any: its keys are added up where they are used
    uint32_t place, limit;
    float scale;                 // 1 / (1 - p)
    bool on;
};
__device__ __forceinline__ RandomKeys device_keys(const Drop &d) {
    return random_keys(d.seed + (d.seed_device != nullptr ? static_cast<uint64_t>(__ldg(d.seed_device)) : 0));
}

// The words of N elements (1, 4 or 8) from the group (low, high) on; N 1: of the one at place `i` of the group.  Drawn before the
// elements are waited for, they fill the time that memory takes.
template <int N>
__device__ __forceinline__ void draw(const Drop &d, const RandomKeys &k, uint32_t low, uint32_t high, uint32_t i, uint32_t *words) {
    if constexpr (N == 1) {
        const uint4 w = random_words(k, low, high, d.place);
        words[0] = i < 2 ? (i == 0 ? w.x : w.y) : (i == 2 ? w.z : w.w);
    } else {
#pragma unroll
        for (int e = 0; e < N; e += 4) {
            const uint4 w = random_words(k, low + e / 4, high, d.place);   // (8 elements from a multiple of 8 on share `high`)
            words[e] = w.x; words[e + 1] = w.y; words[e + 2] = w.z; words[e + 3] = w.w;
        }
    }
}
// v[e]: scaled where kept, else 0.
template <int N>
__device__ __forceinline__ void drop(const Drop &d, const uint32_t *words, float *v) {
#pragma unroll
    for (int e = 0; e < N; ++e) v[e] = words[e] >= d.limit ? v[e] * d.scale : 0.0f;
}

}  // namespace fewbit
