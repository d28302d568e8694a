// Attention for the tensor cores of sm_100a: forward, and a backward pass that recomputes the probabilities.
//
// Mathematics, one head, rows i and keys j, c = scale:
//   S = c Q K^T,  P = exp(S - lse),  O = P V            lse_i = log sum_j exp(S_ij)
//   delta_i = dO_i . O_i,  dV = P^T dO,  dP = dO V^T,  dS = P (dP - delta),  dQ = c dS K,  dK = c dS^T Q
//
// Every kernel has the same roles: warps 0-15 do the element-wise work (a thread owns a row of 128 and a quarter or
// half of a tile's columns), warp 16 issues tcgen05.mma, warp 17 the TMA loads.
// Tiles are 128 x 128; the second operand of a "columns" product is the same shared-memory tile that served the
// "rows" product, read the other way round, and its first operand (P or dS, rounded to 16 bits) goes through
// tensor memory, so no tile of element-wise results ever touches shared memory.
//
//   forward   two row tiles a CTA: one tile's softmax runs while the other's products do
//   dQ        one row tile against all keys: S, dP, dQ (3 products); writes the rows' -lse and -delta for the next kernel
//   dK, dV    one key tile against all rows of all query heads that share it: S^T, dP^T, dV, dK (4 products)
// Where there are few tiles, a cluster of CTAs shares each of them: the tiles of the long axis are dealt out in turn, and
// the sums are joined through distributed shared memory, in a fixed order.
// S and dP are computed in both backward kernels (7 products where 5 would do): in exchange nothing is added
// with atomics, so no binary32 copy of dQ is zeroed, summed and converted, and results are the same every time.
//
// A 128 x 128 x 128 product takes 512 clocks of the tensor cores, 16384 exponentials 1024 of the exponential unit; a
// quarter of the latter are computed on the FMA pipe instead.
#pragma once

#include <climits>
#include <cmath>
#include <type_traits>

#include "fewbit_device.cuh"
#include "fewbit_tensor_core.cuh"

namespace fewbit {
namespace attn {

using namespace tc;

constexpr int kTile = 128;
constexpr int kThreadsAttn = 640;      // five warpgroups: four element-wise ones, and the MMA and load warps (two idle ones fill it up)
constexpr int kMmaWarp = 16, kLoadWarp = 17;
constexpr int kWorkThreads = 512;
// Registers of the element-wise and the issuing threads.  96 a thread at launch: 512 x 104 + 128 x 64 = 512 x 112 + 128 x 32 =
// 61440 = 640 x 96
constexpr int kFwdWork = 112, kFwdIssue = 32, kDqWork = 104, kDqIssue = 64, kDkvWork = 112, kDkvIssue = 32;
constexpr float kLog2e = 1.4426950408889634f;
constexpr uint32_t kNan = 0x7fc00000u;
constexpr int kStatBytes = 2 * kTile * 4;   // a row tile's -lse * log2(e) and -delta

struct Rows {                         // an output tensor
    void *p;
    long long b, i, h;                // strides in elements
};
struct Params {
    CUtensorMap q, k, v, g;           // g: the gradient of the output
    Rows out, o, go, kin, dq, dk, dv; // o, go: outputs and their gradients, read row by row for delta; kin: k, read row by row
    float *lse, *stat;                // stat: a block of kStatBytes for each row tile
    const int *q_offsets, *k_offsets;
    unsigned int *timeouts;
    long long q_rows, k_rows;
    int batch, heads, kv_heads, group, dim;
    int q_len, k_len;                 // of every sequence, or the most of any
    int tiles;                        // row or key tiles (of the kernel's size) in q_len or k_len
    int split;                        // CTAs of a cluster that share a row tile's keys, or a key tile's rows (dK, dV)
    int sms;                          // (the host's)
    bool causal;
    bool after_dq;                    // dK, dV: launched right behind the dQ kernel, whose start is all that its CTAs have waited for
    float scale, scale_log2;          // scale * log2(e)
};

// What one CTA works on.
struct Work {
    int tile, head, batch;
    int q_len, k_len, q_first, k_first;   // lengths, and first rows in the tensors (packed sequences)
    int q_batch;                          // batch coordinate of the tensor maps
    bool packed;
};

// `block`: the CTA's (or its cluster's) place in the grid.  Packed sequences have one more "sequence", number
// `batch`: the rows that belong to none.
__device__ __forceinline__ Work find_work(const Params &p, int block, int heads, bool last_first) {
    Work w;
    w.packed = p.q_offsets != nullptr;
    const int pairs = heads * (p.batch + (w.packed ? 1 : 0));
    const int t = block / pairs, rest = block % pairs;
    w.tile = last_first ? p.tiles - 1 - t : t;
    w.head = rest % heads;
    w.batch = rest / heads;
    w.q_len = p.q_len;
    w.k_len = p.k_len;
    w.q_first = w.k_first = 0;
    w.q_batch = w.batch;
    if (w.packed && w.batch == p.batch) return w;
    if (w.packed) {                   // offsets outside the tensors are cut to them: no access depends on their being right
        const long long q0 = min(max(static_cast<long long>(p.q_offsets[w.batch]), 0ll), p.q_rows);
        const long long q1 = min(max(static_cast<long long>(p.q_offsets[w.batch + 1]), q0), p.q_rows);
        const long long k0 = min(max(static_cast<long long>(p.k_offsets[w.batch]), 0ll), p.k_rows);
        const long long k1 = min(max(static_cast<long long>(p.k_offsets[w.batch + 1]), k0), p.k_rows);
        w.q_first = uniform(static_cast<int>(q0));
        w.k_first = uniform(static_cast<int>(k0));
        w.q_len = uniform(static_cast<int>(min(q1 - q0, static_cast<long long>(p.q_len))));
        w.k_len = uniform(static_cast<int>(min(k1 - k0, static_cast<long long>(p.k_len))));
        w.q_batch = 0;
    }
    return w;
}

// Key tiles that rows [first, last] of a sequence see any key of.
__device__ __forceinline__ int key_tiles(const Params &p, const Work &w, int last) {
    int keys = w.k_len;
    if (p.causal) keys = min(keys, max(0, last + 1 + w.k_len - w.q_len));
    return (keys + kTile - 1) / kTile;
}

// How many of n tiles fall to CTA `rank` of `split` that take them in turn.
__device__ __forceinline__ int share_of(int n, int rank, int split) { return (n - rank + split - 1) / split; }

// Shared memory: tiles first (1 KB aligned), then the barriers.
struct Sync {
    unsigned long long bar[28];
    uint32_t tmem;
    int stop;
};

// A tile of `rows` valid rows: the rest may hold another sequence's values, which a zero probability does not
// silence when they are not finite.  One warp clears them.
template <int HALVES>
__device__ __forceinline__ void clear_rows(uint32_t tile, int rows) {
    const int lane = threadIdx.x & 31;
#pragma unroll
    for (int h = 0; h < HALVES; ++h)
        for (int at = rows * 128 + lane * 16; at < static_cast<int>(kHalfTile); at += 512)
            asm volatile("st.shared.v4.u32 [%0], {%1,%1,%1,%1};" :: "r"(tile + h * kHalfTile + at), "r"(0u) : "memory");
    asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
    __syncwarp();
}

template <int HALVES>
__device__ __forceinline__ void load_halves(uint32_t dst, const CUtensorMap *map, int row, int head, int batch, uint32_t bar) {
#pragma unroll
    for (int h = 0; h < HALVES; ++h) load_tile(dst + h * kHalfTile, map, 64 * h, row, head, batch, bar);
}

// N values of one row, scaled and rounded, to columns [col, col + N) of a tensor of `dim` columns.
template <typename T, int N>
__device__ __forceinline__ void store_columns(T *row, int col, int dim, const uint32_t *r, float factor) {
#pragma unroll
    for (int c = 0; c < N; c += 8) {
        if (col + c >= dim) break;                                    // dim is a multiple of 8
        uint4 v;
        v.x = pack2<T>(__uint_as_float(r[c]) * factor, __uint_as_float(r[c + 1]) * factor);
        v.y = pack2<T>(__uint_as_float(r[c + 2]) * factor, __uint_as_float(r[c + 3]) * factor);
        v.z = pack2<T>(__uint_as_float(r[c + 4]) * factor, __uint_as_float(r[c + 5]) * factor);
        v.w = pack2<T>(__uint_as_float(r[c + 6]) * factor, __uint_as_float(r[c + 7]) * factor);
        *reinterpret_cast<uint4 *>(row + col + c) = v;
    }
}
template <typename T>
__device__ __forceinline__ void zero_columns(T *row, int dim) {
    for (int c = 0; c < dim; c += 8) *reinterpret_cast<uint4 *>(row + c) = make_uint4(0, 0, 0, 0);
}

__device__ __forceinline__ long long row_of(const Work &w, const Rows &t, int head, int i, int first) {
    return (w.packed ? 0 : w.batch * t.b) + (static_cast<long long>(first) + i) * t.i + head * t.h;
}
// Block of a row tile in `stat`: (batch, heads, tiles), or (heads, rows / 128 + sequences + 1) for packed sequences, whose
// tile t starts at block first / 128 + sequence (a sequence has at most one tile more than whole tiles of rows).
__device__ __forceinline__ float *stat_block(const Params &p, const Work &w, int head, int tile) {
    const long long at = w.packed ? static_cast<long long>(head) * (p.q_rows / kTile + p.batch + 1) + w.q_first / kTile + w.batch + tile
                                  : (static_cast<long long>(w.batch) * p.heads + head) * ((p.q_len + kTile - 1) / kTile) + tile;
    return p.stat + at * (kStatBytes / 4);
}
// Packed sequences: rows in front of the first and behind the last one, and those of a sequence past the bound of its
// length, are zero in every output, their lse -inf.  The CTAs of the extra sequence share them.
template <typename T>
__device__ __forceinline__ void fill_outside(const Params &p, const Work &w, const int *offsets, long long rows, int longest, const Rows &t, float *lse) {
    auto clear = [&](long long row) {
        zero_columns<T>(static_cast<T *>(t.p) + row * t.i + w.head * t.h, p.dim);
        if (lse != nullptr) lse[static_cast<long long>(w.head) * rows + row] = -INFINITY;
    };
    const long long start = static_cast<long long>(w.tile) * kThreadsAttn + threadIdx.x, step = static_cast<long long>(p.tiles) * kThreadsAttn;
    const long long first = min(max(static_cast<long long>(offsets[0]), 0ll), rows);
    const long long last = min(max(static_cast<long long>(offsets[p.batch]), first), rows);
    for (long long i = start; i < first + rows - last; i += step) clear(i < first ? i : last + (i - first));
    for (long long b = start; b < p.batch; b += step) {               // a thread for each sequence: longer ones than announced are rare
        const long long from = min(max(static_cast<long long>(offsets[b]), 0ll), rows), end = min(static_cast<long long>(offsets[b + 1]), rows);
        for (long long i = from + longest; i < end; ++i) clear(i);
    }
}

// Place of a row's lse: (batch, heads, q_len), or (heads, rows) for packed sequences.
__device__ __forceinline__ long long stat_of(const Params &p, const Work &w, int head, int i) {
    return w.packed ? static_cast<long long>(head) * p.q_rows + w.q_first + i
                    : (static_cast<long long>(w.batch) * p.heads + head) * p.q_len + i;
}

__device__ __forceinline__ bool stopped(const Sync *sync) { return *reinterpret_cast<const volatile int *>(&sync->stop) != 0; }

__device__ __forceinline__ uint32_t start_cta(Sync *sync, int barriers, const uint32_t *counts) {
    if (threadIdx.x == 0) {
        sync->stop = 0;
        for (int i = 0; i < barriers; ++i) barrier_init(smem_address(&sync->bar[i]), counts[i]);
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    if (threadIdx.x / 32 == kMmaWarp) tmem_alloc(smem_address(&sync->tmem), 512);
    fence_before();
    __syncthreads();
    fence_after();
    return uniform(*reinterpret_cast<volatile uint32_t *>(&sync->tmem));
}
// Every role is through: nothing is in flight any more.
__device__ __forceinline__ void end_cta(uint32_t tmem) {
    fence_before();
    __syncthreads();
    fence_after();
    if (threadIdx.x / 32 == kMmaWarp) tmem_free(tmem, 512);
}

// ---------------------------------------------------------------------------------------------------
// forward
// ---------------------------------------------------------------------------------------------------
// One pass over the keys with a running reference and sum of the softmax (Milakov and Gimelshein, Online normalizer calculation
// for softmax, 2018; that the reference may stay while it does no harm, and that a share of the exponentials may be computed by a
// polynomial, is known from later published work on attention).  For each pair of row tiles and key tile: 2048
// clocks of products, 2048 of exponentials (of which a quarter goes elsewhere), 64 KB from L2.  Two row tiles share every
// K and V tile that is loaded, and each one's softmax runs while the other's products do.  Measured, bfloat16, heads of
// 128, causal: 16384 rows, 8 heads on 2, 484 us = 1.14 PFLOP/s, 68 % of a burst of matrix products and 81 % of what they
// sustain: the power limit holds the SMs at 1.6 GHz there; 4 x 2048 rows, 16 heads on 4, 89 us = 0.77 PFLOP/s: 512 CTAs of
// 2 to 16 key tiles, each with a start and an end that no product covers.  One row on 8192 keys: 25 us, 8 tiles one
// after another in each of 64 CTAs and the joining of their sums.
// Barriers: q (2 row tiles), k full/empty (2 stages), v full/empty, S full (2), the first half of each thread's part of P
// ready (2), all of it (2), O done (2), drained.
enum { fQ = 0, fKFull = 2, fKEmpty = 4, fVFull = 6, fVEmpty = 8, fS = 10, fP = 12, fPEnd = 14, fO = 16, fDrain = 18, fBars = 19 };

template <int DIM> constexpr int fwd_smem() { return 6 * (DIM / 64) * static_cast<int>(kHalfTile) + 1024 + static_cast<int>(sizeof(Sync)) + 8 * kTile * 4; }

// Barriers of two warps.
__device__ __forceinline__ void pair_barrier(int id) { asm volatile("bar.sync %0, 64;" :: "r"(id) : "memory"); }
__device__ __forceinline__ bool pair_any(int id, bool x) {
    uint32_t any;
    asm volatile("{\n.reg .pred p, q;\nsetp.ne.u32 p, %1, 0;\nbarrier.cta.red.or.pred q, %2, 64, p;\nselp.u32 %0, 1, 0, q;\n}"
                 : "=r"(any) : "r"(static_cast<uint32_t>(x)), "r"(id) : "memory");
    return any != 0;
}

// 32 columns of a row: probabilities, rounded to `s_at`, and their sum.  MIXED: a quarter of them on the FMA pipe.
template <typename T, bool MIXED>
__device__ __forceinline__ void fwd_probabilities(const uint32_t *s, float scale, float shift, float (&part)[4], uint32_t at) {
    uint32_t r[16];
#pragma unroll
    for (int e = 0; e < 16; ++e) {
        float a, b;
        if (MIXED && e % 4 == 3) exp2_scaled<true>(a, b, __uint_as_float(s[2 * e]), __uint_as_float(s[2 * e + 1]), scale, shift, shift);
        else exp2_scaled<false>(a, b, __uint_as_float(s[2 * e]), __uint_as_float(s[2 * e + 1]), scale, shift, shift);
        add2(part[2 * (e & 1)], part[2 * (e & 1) + 1], part[2 * (e & 1)], part[2 * (e & 1) + 1], a, b);
        r[e] = pack2<T>(a, b);
    }
    tmem_st16(at, r);
}

template <typename T, int DIM>
__global__ void __launch_bounds__(kThreadsAttn, 1)
attention_fwd_kernel(const __grid_constant__ Params p) {
    constexpr int HALVES = DIM / 64;
    constexpr uint32_t kBytes = HALVES * kHalfTile;                   // of one tile
    extern __shared__ uint8_t raw[];
    const uint32_t base = (smem_address(raw) + 1023u) & ~1023u;
    Sync *sync = reinterpret_cast<Sync *>(raw + (base - smem_address(raw)) + 6 * kBytes);
    float *exchange = reinterpret_cast<float *>(sync + 1);            // [row tile][half][128]
    float *joined = exchange + 4 * kTile;                             // [row tile][reference, sum][128], for the cluster
    const int warp = uniform(static_cast<int>(threadIdx.x >> 5)), lane = threadIdx.x & 31;
    pdl_wait();
    const int rank = p.split > 1 ? static_cast<int>(cluster_rank()) : 0;
    const Work w = find_work(p, blockIdx.x / p.split, p.heads, true);
    if (w.packed && w.batch == p.batch) {                             // (the whole cluster)
        if (rank == 0) fill_outside<T>(p, w, p.q_offsets, p.q_rows, p.q_len, p.out, p.lse);
        return;
    }
    const int q0 = w.tile * 2 * kTile;
    if (q0 >= w.q_len) return;                                        // packed: a shorter sequence
    const int kv_head = w.head / p.group;
    // key tiles of each row tile (0 also for a row tile past the end)
    // that fall to this CTA: number rank, rank + split, ...
    const int n0 = uniform(share_of(key_tiles(p, w, min(q0 + kTile, w.q_len) - 1), rank, p.split));
    const int n1 = uniform(share_of(q0 + kTile < w.q_len ? key_tiles(p, w, min(q0 + 2 * kTile, w.q_len) - 1) : 0, rank, p.split));
    auto key_tile = [&](int j) { return rank + j * p.split; };
    const int n = max(n0, n1);

    constexpr uint32_t counts[fBars] = {1, 1, 1, 1, 1, 1, 1, 1, 1, 1, 1, 1, 8, 8, 8, 8, 1, 1, 1};
    const uint32_t tmem = start_cta(sync, fBars, counts);
    auto bar = [&](int i) { return smem_address(&sync->bar[i]); };
    auto wait = [&](int i, uint32_t parity) { return barrier_wait(bar(i), parity, &sync->stop, p.timeouts); };
    const uint32_t sm_q = base, sm_k = base + 2 * kBytes, sm_v = base + 4 * kBytes;
    // tensor memory: S of both row tiles (each 32 columns of P in the first half of the scores that they came from), then O of both
    const uint32_t tm_s = tmem, tm_o = tmem + 2 * kTile;

    if (warp >= kMmaWarp) {
        give_registers<kFwdIssue>();
        if (warp == kLoadWarp) {
            int issued_k = 0, issued_v = 0;
            if (n > 0 && lane == 0) {
                prefetch_map(&p.q);
                prefetch_map(&p.k);
                prefetch_map(&p.v);
                barrier_expect(bar(fQ), kBytes);
                load_halves<HALVES>(sm_q, &p.q, w.q_first + q0, w.head, w.q_batch, bar(fQ));
                if (n1 > 0) {
                    barrier_expect(bar(fQ + 1), kBytes);
                    load_halves<HALVES>(sm_q + kBytes, &p.q, w.q_first + q0 + kTile, w.head, w.q_batch, bar(fQ + 1));
                }
            }
            for (int j = 0; j < n; ++j) {
                const int s = j & 1;
                const uint32_t again = ((j >> 1) & 1) ^ 1;            // the stage's previous tile has been used
                if (!wait(fKEmpty + s, again)) break;
                if (lane == 0) {
                    barrier_expect(bar(fKFull + s), kBytes);
                    load_halves<HALVES>(sm_k + s * kBytes, &p.k, w.k_first + key_tile(j) * kTile, kv_head, w.q_batch, bar(fKFull + s));
                }
                issued_k = j + 1;
                if (!wait(fVEmpty + s, again)) break;
                if (lane == 0) {
                    barrier_expect(bar(fVFull + s), kBytes);
                    load_halves<HALVES>(sm_v + s * kBytes, &p.v, w.k_first + key_tile(j) * kTile, kv_head, w.q_batch, bar(fVFull + s));
                }
                issued_v = j + 1;
            }
            if (stopped(sync)) {                                      // given up somewhere: let the copies land before the CTA ends
                if (n > 0) barrier_wait(bar(fQ), 0, nullptr, p.timeouts);
                if (n1 > 0) barrier_wait(bar(fQ + 1), 0, nullptr, p.timeouts);
                for (int s = 0; s < 2; ++s) {
                    if (issued_k > s) barrier_wait(bar(fKFull + s), ((issued_k - 1 - s) >> 1) & 1, nullptr, p.timeouts);
                    if (issued_v > s) barrier_wait(bar(fVFull + s), ((issued_v - 1 - s) >> 1) & 1, nullptr, p.timeouts);
                }
            }
        } else if (warp == kMmaWarp) {
            const uint32_t leader = elect_leader();
            auto scores = [&](int t, int j) {                         // S of row tile t against key tile j
                product_rows<T, DIM>(leader, tm_s + t * kTile, sm_q + t * kBytes, sm_k + (j & 1) * kBytes);
                commit(leader, bar(fS + t));
            };
            bool ok = n == 0 || (wait(fQ, 0) && (n1 == 0 || wait(fQ + 1, 0)) && wait(fKFull, 0));
            if (ok && n > 0) {
                fence_after();
                if (n0 > 0) scores(0, 0);
                if (n1 > 0) scores(1, 0);
                commit(leader, bar(fKEmpty));
            }
            for (int j = 0; ok && j < n; ++j) {
                ok = wait(fVFull + (j & 1), (j >> 1) & 1) && (j + 1 >= n || wait(fKFull + ((j + 1) & 1), ((j + 1) >> 1) & 1));
                if (!ok) break;
                if (w.packed && (key_tile(j) + 1) * kTile > w.k_len) clear_rows<HALVES>(sm_v + (j & 1) * kBytes, w.k_len - key_tile(j) * kTile);
                for (int t = 0; t < 2 && ok; ++t) {
                    const int nt = t ? n1 : n0;
                    if (j >= nt) continue;
                    const uint32_t at = tm_s + t * kTile;
                    // the product starts on one half of P while the other is computed
                    ok = wait(fP + t, j & 1);
                    if (!ok) break;
                    fence_after();
                    product_columns<T, DIM, 2, 32, 0xcc>(leader, tm_o + t * kTile, at, sm_v + (j & 1) * kBytes, j > 0);
                    ok = wait(fPEnd + t, j & 1);
                    if (!ok) break;
                    fence_after();
                    product_columns<T, DIM, 2, 32, 0x33>(leader, tm_o + t * kTile, at, sm_v + (j & 1) * kBytes, true);
                    commit(leader, bar(fO + t));
                    if (j + 1 < nt) scores(t, j + 1);
                }
                commit(leader, bar(fVEmpty + (j & 1)));
                if (j + 1 < n) commit(leader, bar(fKEmpty + ((j + 1) & 1)));
            }
            commit(leader, bar(fDrain));
            barrier_wait(bar(fDrain), 0, nullptr, p.timeouts);
        }
        if (p.split > 1) {                                            // the element-wise warps' two barriers, below
            cluster_sync();
            cluster_sync();
        }
    } else {
        take_registers<kFwdWork>();
        const int t = warp >> 3, half = (warp >> 2) & 1;              // row tile; columns [64 half, 64 half + 64) of every key tile
        const int nt = t ? n1 : n0, r = threadIdx.x & 127;
        const int i = q0 + t * kTile + r;                             // this thread's row
        const uint32_t my_lane = static_cast<uint32_t>(warp & 3) << 21;
        const uint32_t s_at = tm_s + t * kTile + 64 * half + my_lane, o_at = tm_o + t * kTile + half * (DIM / 2) + my_lane;
        const int pair = 1 + 4 * t + (warp & 3);                      // barrier of the two warps that share their rows
        float *mine = exchange + (2 * t + half) * kTile + r, *other = exchange + (2 * t + 1 - half) * kTile + r;
        // the row sees keys [0, seen)
        const int seen = p.causal ? min(w.k_len, i + 1 + w.k_len - w.q_len) : w.k_len;
        const int tile_seen = p.causal ? min(w.k_len, q0 + t * kTile + 1 + w.k_len - w.q_len) : w.k_len;   // by its first row
        float top = -INFINITY, sum = 0.0f;                            // of the raw products; the sum of this thread's columns
        bool ok = true;
        for (int j = 0; j < nt; ++j) {
            ok = wait(fS + t, j & 1);                                 // (a wait given up ends the loop below, for all threads of the tile)
            fence_after();
            const bool edge = (key_tile(j) + 1) * kTile > tile_seen;
            const int limit = seen - key_tile(j) * kTile - 64 * half;
            // Scores are read twice, 32 columns at a time, for the maximum and for the probabilities: reading them costs less
            // than holding 64 of them in registers.
            uint32_t s[32];
            auto read = [&](int c) {
                tmem_ld32(s_at + 32 * c, s);
                wait_ld(s);
                if (edge) {
#pragma unroll
                    for (int e = 0; e < 32; ++e) s[e] = 32 * c + e < limit ? s[e] : 0xff800000u;
                }
            };
            float best[4] = {-INFINITY, -INFINITY, -INFINITY, -INFINITY};
            auto maximum = [&]() {
#pragma unroll
                for (int e = 0; e < 32; e += 2)                       // two at a time: a three-operand maximum
                    best[(e >> 1) & 3] = max3_nan(best[(e >> 1) & 3], __uint_as_float(s[e]), __uint_as_float(s[e + 1]));
            };
            read(0);
            maximum();
            read(1);
            maximum();
            const float high = max3_nan(max3_nan(best[0], best[1], best[2]), best[3], best[3]);
            // The sums' reference moves only when a product passes it by 2^8: until then probabilities up to 2^8
            // are held, which cost no precision, and O needs no rescaling.  The row's two threads move it together: whether
            // any row of their two warps moves is one barrier, and only then they exchange their maxima.  A score that is NaN
            // becomes the reference, and with it the whole row.
            auto moves = [&](float to) { return to != top && !((to - top) * p.scale_log2 <= 8.0f); };
            const bool above = moves(high);
            if (pair_any(pair, above || !ok)) {
                if (pair_any(pair, !ok)) {
                    ok = false;
                    break;
                }
                *mine = high;
                pair_barrier(pair);
                const float row_high = max3_nan(high, *other, high);
                const bool move = moves(row_high);
                const float next = move ? row_high : top;
                const float factor = move ? exp2_fast((top - next) * p.scale_log2) : 1.0f;
                top = next;
                sum *= factor;
                if (j > 0) {
                    ok = wait(fO + t, (j - 1) & 1);
                    if (pair_any(pair, !ok)) {
                        ok = false;
                        break;
                    }
                    fence_after();
#pragma unroll
                    for (int c = 0; c < DIM / 64; ++c) {
                        uint32_t o[32];
                        tmem_ld32(o_at + 32 * c, o);
                        wait_ld(o);
#pragma unroll
                        for (int e = 0; e < 32; ++e) o[e] = __float_as_uint(__uint_as_float(o[e]) * factor);
                        tmem_st32(o_at + 32 * c, o);
                    }
                }
            }
            const float shift = top == -INFINITY ? 0.0f : -top * p.scale_log2;
            float part[4] = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
            for (int c = 1; c >= 0; --c) {                            // (columns 32 to 63 are still there)
                if (c == 0) read(0);
                if (edge) fwd_probabilities<T, false>(s, p.scale_log2, shift, part, s_at + 32 * c);
                else fwd_probabilities<T, true>(s, p.scale_log2, shift, part, s_at + 32 * c);
                wait_st();
                fence_before();
                __syncwarp();
                if (lane == 0) barrier_arrive(bar((c == 1 ? fP : fPEnd) + t));
            }
            sum += (part[0] + part[1]) + (part[2] + part[3]);
        }
        if (nt > 0 && ok) ok = wait(fO + t, (nt - 1) & 1);
        fence_after();
        if (!ok) sum = NAN;                                           // given up: out and lse say so
        *mine = sum;                                                  // (the last exchange of maxima was read before P was ready)
        pair_barrier(pair);
        sum += *other;
        const bool live = i < w.q_len;
        T *row = static_cast<T *>(p.out.p) + (live ? row_of(w, p.out, w.head, i, w.q_first) : 0);
        if (p.split == 1) {
            if (nt > 0) {
                const float factor = sum > 0.0f || sum != sum ? 1.0f / sum : 0.0f;
#pragma unroll
                for (int c = 0; c < DIM / 64; ++c) {
                    uint32_t o[32];
                    tmem_ld32(o_at + 32 * c, o);
                    wait_ld(o);
                    if (live) store_columns<T, 32>(row, half * (DIM / 2) + 32 * c, p.dim, o, factor);
                }
            } else if (live && half == 0) {
                zero_columns<T>(row, p.dim);
            }
            if (live && half == 0) p.lse[stat_of(p, w, w.head, i)] = sum == 0.0f ? -INFINITY : top * p.scale + logf(sum);
        } else {
            // Every CTA lays its O, reference and sum of each row out in shared memory, [row tile][column][row]; a share of the
            // columns is brought to the largest reference, added up and divided by each.
            // (The tiles that this overwrites are the other row tile's too, which may see more keys: all its products first.)
            asm volatile("bar.sync 9, %0;" :: "n"(kWorkThreads) : "memory");
            const uint32_t mine_o = base + static_cast<uint32_t>(t * DIM) * (kTile * 4) + r * 4;
            const uint32_t mine_stat = smem_address(joined + 2 * t * kTile + r);
#pragma unroll
            for (int c = 0; c < DIM / 64; ++c) {
                uint32_t o[32];
                tmem_ld32(o_at + 32 * c, o);                          // (what it holds does not matter where there was no key tile)
                wait_ld(o);
#pragma unroll
                for (int e = 0; e < 32; ++e)
                    asm volatile("st.shared.u32 [%0], %1;" :: "r"(mine_o + (half * (DIM / 2) + 32 * c + e) * (kTile * 4)), "r"(nt > 0 ? o[e] : 0u) : "memory");
            }
            if (half == 0) {
                joined[2 * t * kTile + r] = top;
                joined[(2 * t + 1) * kTile + r] = sum;
            }
            cluster_sync();
            float high = -INFINITY, total = 0.0f;
            for (int k = 0; k < p.split; ++k) high = fmaxf(high, load_peer(mine_stat, k));
            const float reference = high == -INFINITY ? 0.0f : high * p.scale_log2;
            for (int k = 0; k < p.split; ++k) total += exp2_fast(load_peer(mine_stat, k) * p.scale_log2 - reference) * load_peer(mine_stat + kTile * 4, k);
            const float factor = total > 0.0f || total != total ? 1.0f / total : 0.0f;
            const int share = DIM / p.split;                          // a multiple of 16
            for (int col = rank * share + half * (share / 2); col < rank * share + (half + 1) * (share / 2); col += 8) {
                float v[8] = {0.0f, 0.0f, 0.0f, 0.0f, 0.0f, 0.0f, 0.0f, 0.0f};
                for (int k = 0; k < p.split; ++k) {
                    const float weight = exp2_fast(load_peer(mine_stat, k) * p.scale_log2 - reference);
                    float x[8];
#pragma unroll
                    for (int e = 0; e < 8; ++e) x[e] = load_peer(mine_o + (col + e) * (kTile * 4), k);
#pragma unroll
                    for (int e = 0; e < 8; ++e) v[e] = fmaf(weight, x[e], v[e]);
                }
                uint32_t o[8];
#pragma unroll
                for (int e = 0; e < 8; ++e) o[e] = __float_as_uint(v[e]);
                if (live) store_columns<T, 8>(row, col, p.dim, o, factor);
            }
            if (live && half == 0 && rank == 0) p.lse[stat_of(p, w, w.head, i)] = total == 0.0f ? -INFINITY : high * p.scale + logf(total);
            cluster_sync();                                           // nobody's shared memory goes before it has been read
        }
    }
    end_cta(tmem);
}

// ---------------------------------------------------------------------------------------------------
// backward, dQ (and the rows' statistics)
// ---------------------------------------------------------------------------------------------------
// Three products (1536 clocks) and 1024 of exponentials for each row and key tile, which loads 64 KB for the one row tile
// that tensor and shared memory have room for: 37 bytes a clock into each SM are what L2 gives when all SMs ask, so the loads
// take 1750 clocks and bound it.  Tensor pipe 42 % active on 4 x 2048 rows, 16 heads on 4, causal; the whole backward pass
// takes 275 us there (0.62 PFLOP/s counting five products, 0.87 counting the seven that are computed), and 1.61 ms for
// 16384 rows, 8 heads on 2 (0.85 and 1.18 PFLOP/s, the latter 84 % of what matrix products sustain at the power limit).
// Barriers: q and g, k full/empty (3 stages: a tile is used twice, one iteration apart), v full/empty (2 stages), S full (2),
// dP full, dS ready, dQ done.
enum { qQ = 0, qKFull = 1, qKEmpty = 4, qVFull = 7, qVEmpty = 9, qS = 11, qDp = 13, qDs = 14, qDone = 15, qBars = 16 };

template <int DIM> constexpr int dq_smem() { return 7 * (DIM / 64) * static_cast<int>(kHalfTile) + static_cast<int>(sizeof(Sync)) + 5 * kTile * 4; }

template <typename T, int DIM>
__global__ void __launch_bounds__(kThreadsAttn, 1)
attention_dq_kernel(const __grid_constant__ Params p) {
    constexpr int HALVES = DIM / 64;
    constexpr uint32_t kBytes = HALVES * kHalfTile;
    extern __shared__ __align__(1024) uint8_t raw[];
    const uint32_t base = smem_address(raw);                          // (its declaration aligns it: there is no room to do it here)
    Sync *sync = reinterpret_cast<Sync *>(raw + 7 * kBytes);
    float *row_delta = reinterpret_cast<float *>(sync + 1);           // [128]
    float *row_sum = row_delta + kTile;                               // [4][128]
    const int warp = uniform(static_cast<int>(threadIdx.x >> 5)), lane = threadIdx.x & 31;
    pdl_wait();
    pdl_launch_dependents();                                          // the dK and dV kernel may set itself up
    const int rank = p.split > 1 ? static_cast<int>(cluster_rank()) : 0;
    const Work w = find_work(p, blockIdx.x / p.split, p.heads, true);
    if (w.packed && w.batch == p.batch) {                             // (the whole cluster)
        if (rank == 0) fill_outside<T>(p, w, p.q_offsets, p.q_rows, p.q_len, p.dq, nullptr);
        return;
    }
    const int q0 = w.tile * kTile;
    if (q0 >= w.q_len) return;
    const int kv_head = w.head / p.group;
    // key tiles that the rows see, and how many of them fall to this CTA: number rank, rank + split, ...
    const int n_all = uniform(key_tiles(p, w, min(q0 + kTile, w.q_len) - 1));
    const int n = share_of(n_all, rank, p.split);
    auto key_tile = [&](int j) { return rank + j * p.split; };

    // The outputs that delta needs, read while the CTA sets itself up: DIM / 8 lanes a row, 8 rows for each warp.  (From here on
    // the L2's bandwidth is the tiles' that are on their way.)
    constexpr int kLanes = DIM / 8, kRows = 32 / kLanes;
    uint4 outputs[8 / kRows];
    float lse = -INFINITY;
    if (warp < kMmaWarp) {
#pragma unroll
        for (int x = 0; n > 0 && n_all > 1 && x < 8 / kRows; ++x) {
            const int row = q0 + 8 * warp + kRows * x + lane / kLanes, col = lane % kLanes * 8;
            const bool there = row < w.q_len && col < p.dim;
            const T *from = static_cast<const T *>(p.o.p) + row_of(w, p.o, w.head, there ? row : 0, w.q_first) + (there ? col : 0);
            outputs[x] = there ? __ldg(reinterpret_cast<const uint4 *>(from)) : make_uint4(0, 0, 0, 0);
        }
        const int row = q0 + (threadIdx.x & 127);
        if (row < w.q_len) lse = p.lse[stat_of(p, w, w.head, row)];
    }

    constexpr uint32_t counts[qBars] = {1, 1, 1, 1, 1, 1, 1, 1, 1, 1, 1, 1, 1, 1, 16, 1};
    const uint32_t tmem = start_cta(sync, qBars, counts);
    auto bar = [&](int i) { return smem_address(&sync->bar[i]); };
    auto wait = [&](int i, uint32_t parity) { return barrier_wait(bar(i), parity, &sync->stop, p.timeouts); };
    const uint32_t sm_q = base, sm_g = base + kBytes, sm_k = base + 2 * kBytes, sm_v = base + 5 * kBytes;
    // tensor memory: S twice (dS takes its place), dP, dQ
    const uint32_t tm_s = tmem, tm_dp = tmem + 2 * kTile, tm_dq = tmem + 3 * kTile;

    if (warp >= kMmaWarp) {
        give_registers<kDqIssue>();
        if (warp == kLoadWarp) {
            int issued_k = 0, issued_v = 0;
            if (n > 0 && lane == 0) {
                prefetch_map(&p.q);
                prefetch_map(&p.k);
                prefetch_map(&p.v);
                prefetch_map(&p.g);
                barrier_expect(bar(qQ), 2 * kBytes);
                load_halves<HALVES>(sm_q, &p.q, w.q_first + q0, w.head, w.q_batch, bar(qQ));
                load_halves<HALVES>(sm_g, &p.g, w.q_first + q0, w.head, w.q_batch, bar(qQ));
            }
            for (int j = 0; j < n; ++j) {
                const int s = j & 1, s3 = j % 3;
                if (!wait(qKEmpty + s3, ((j / 3) & 1) ^ 1)) break;
                if (lane == 0) {
                    barrier_expect(bar(qKFull + s3), kBytes);
                    load_halves<HALVES>(sm_k + s3 * kBytes, &p.k, w.k_first + key_tile(j) * kTile, kv_head, w.q_batch, bar(qKFull + s3));
                }
                issued_k = j + 1;
                if (!wait(qVEmpty + s, ((j >> 1) & 1) ^ 1)) break;
                if (lane == 0) {
                    barrier_expect(bar(qVFull + s), kBytes);
                    load_halves<HALVES>(sm_v + s * kBytes, &p.v, w.k_first + key_tile(j) * kTile, kv_head, w.q_batch, bar(qVFull + s));
                }
                issued_v = j + 1;
            }
            if (stopped(sync)) {
                if (n > 0) barrier_wait(bar(qQ), 0, nullptr, p.timeouts);
                for (int s = 0; s < 3; ++s)
                    if (issued_k > s) barrier_wait(bar(qKFull + s), ((issued_k - 1 - s) / 3) & 1, nullptr, p.timeouts);
                for (int s = 0; s < 2; ++s)
                    if (issued_v > s) barrier_wait(bar(qVFull + s), ((issued_v - 1 - s) >> 1) & 1, nullptr, p.timeouts);
            }
        } else if (warp == kMmaWarp) {
            const uint32_t leader = elect_leader();
            // K tile j is used by S_j and, transposed, by dQ_j; V tile j by dP_j
            auto scores = [&](int j) {
                if (!wait(qKFull + j % 3, (j / 3) & 1)) return false;
                if (w.packed && (key_tile(j) + 1) * kTile > w.k_len) clear_rows<HALVES>(sm_k + (j % 3) * kBytes, w.k_len - key_tile(j) * kTile);
                product_rows<T, DIM>(leader, tm_s + (j & 1) * kTile, sm_q, sm_k + (j % 3) * kBytes);
                commit(leader, bar(qS + (j & 1)));
                return true;
            };
            auto dprobs = [&](int j) {
                if (!wait(qVFull + (j & 1), (j >> 1) & 1)) return false;
                product_rows<T, DIM>(leader, tm_dp, sm_g, sm_v + (j & 1) * kBytes);
                commit(leader, bar(qDp));
                commit(leader, bar(qVEmpty + (j & 1)));
                return true;
            };
            bool ok = n == 0 || (wait(qQ, 0) && scores(0) && dprobs(0) && (n < 2 || scores(1)));
            for (int j = 0; ok && j < n; ++j) {
                ok = wait(qDs, j & 1);                                // dS_j written, dP_j read
                if (!ok) break;
                fence_after();
                if (j + 1 < n && !(ok = dprobs(j + 1))) break;
                const uint32_t at = tm_s + (j & 1) * kTile;
                product_columns<T, DIM, 2, 32>(leader, tm_dq, at, sm_k + (j % 3) * kBytes, j > 0);
                commit(leader, bar(qKEmpty + j % 3));
                if (j + 2 < n) ok = scores(j + 2);                    // over dS_j, after its product
            }
            commit(leader, bar(qDone));
            barrier_wait(bar(qDone), 0, nullptr, p.timeouts);
        }
        if (p.split > 1) {                                            // the element-wise warps' two barriers, below
            cluster_sync();
            cluster_sync();
        }
    } else {
        take_registers<kDqWork>();
        const int part = warp >> 2;                                   // columns [32 part, 32 part + 32) of every tile
        const int r = threadIdx.x & 127, i = q0 + r;
        const bool live = i < w.q_len;
        const uint32_t my_lane = static_cast<uint32_t>(warp & 3) << 21;
        const float minus_lse = lse == -INFINITY ? -INFINITY : -lse * kLog2e;   // a row that sees nothing: every probability is 0
        // delta from the rounded outputs is off by their rounding.  Rows that see few keys feel that most, and those of one key
        // tile (`single`) need no outputs: their delta is the sum of P dP, which is all there before dS is computed.  Longer rows
        // know at the end how far theirs was off, by the sum of dS, which should be 0: dK gets the corrected value.
        const bool single = n_all == 1;
        bool ok = n == 0 || single || wait(qQ, 0);
#pragma unroll
        for (int x = 0; x < 8 / kRows; ++x) {
            const int row = 8 * warp + kRows * x + lane / kLanes;
            float sum = 0.0f;
            if (n > 0 && !single && q0 + row < w.q_len) {
                const uint4 g = tile_chunk(sm_g, row, lane % kLanes);
                T a[8], b[8];
                memcpy(a, &outputs[x], 16);
                memcpy(b, &g, 16);
#pragma unroll
                for (int e = 0; e < 8; ++e) sum = fmaf(load1(&a[e]), load1(&b[e]), sum);
            }
#pragma unroll
            for (int m = kLanes / 2; m > 0; m >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, m);
            if (lane % kLanes == 0) row_delta[row] = sum;
        }
        asm volatile("bar.sync 1, %0;" :: "n"(kWorkThreads) : "memory");   // the element-wise warps only
        float minus_delta = -row_delta[r], drift = 0.0f;
        auto over_parts = [&](float mine) {                           // a row's sum over its four threads
            row_sum[part * kTile + r] = mine;
            asm volatile("bar.sync 1, %0;" :: "n"(kWorkThreads) : "memory");
            return (row_sum[r] + row_sum[kTile + r]) + (row_sum[2 * kTile + r] + row_sum[3 * kTile + r]);
        };
        const int seen = p.causal ? min(w.k_len, i + 1 + w.k_len - w.q_len) : w.k_len;
        const int tile_seen = p.causal ? min(w.k_len, q0 + 1 + w.k_len - w.q_len) : w.k_len;
        for (int j = 0; ok && j < n; ++j) {
            const uint32_t s_at = tm_s + (j & 1) * kTile + 32 * part + my_lane;
            ok = wait(qS + (j & 1), (j >> 1) & 1);
            if (!ok) {
                if (single) over_parts(0.0f);                         // the others wait there
                break;
            }
            fence_after();
            uint32_t s[32], d[32], out[16];
            float prob[32];
            tmem_ld32(s_at, s);
            wait_ld(s);
            const bool edge = (key_tile(j) + 1) * kTile > tile_seen;
            if (edge) {
#pragma unroll
                for (int c = 0; c < 32; c += 2)
                    exp2_scaled<false>(prob[c], prob[c + 1], __uint_as_float(s[c]), __uint_as_float(s[c + 1]), p.scale_log2, minus_lse, minus_lse);
            } else {
#pragma unroll
                for (int c = 0; c < 32; c += 2) {
                    if (c % 8 == 6) exp2_scaled<true>(prob[c], prob[c + 1], __uint_as_float(s[c]), __uint_as_float(s[c + 1]), p.scale_log2, minus_lse, minus_lse);
                    else exp2_scaled<false>(prob[c], prob[c + 1], __uint_as_float(s[c]), __uint_as_float(s[c + 1]), p.scale_log2, minus_lse, minus_lse);
                }
            }
            ok = wait(qDp, j & 1);
            if (!ok) {
                if (single) over_parts(0.0f);
                break;
            }
            fence_after();
            tmem_ld32(tm_dp + 32 * part + my_lane, d);
            wait_ld(d);
            float ds[32];
            const int limit = seen - key_tile(j) * kTile - 32 * part;           // places from here on the row does not see, whatever they hold
            if (single) {
                float sum = 0.0f;
#pragma unroll
                for (int c = 0; c < 32; ++c) {
                    ds[c] = c < limit ? prob[c] * __uint_as_float(d[c]) : 0.0f;
                    sum += ds[c];
                }
                minus_delta = -over_parts(sum);
#pragma unroll
                for (int c = 0; c < 32; ++c) ds[c] = c < limit ? fmaf(prob[c], minus_delta, ds[c]) : 0.0f;
            } else {
#pragma unroll
                for (int c = 0; c < 32; c += 2) {
                    add2(ds[c], ds[c + 1], __uint_as_float(d[c]), __uint_as_float(d[c + 1]), minus_delta, minus_delta);
                    mul2(ds[c], ds[c + 1], ds[c], ds[c + 1], prob[c], prob[c + 1]);
                }
                if (edge) {
#pragma unroll
                    for (int c = 0; c < 32; ++c) ds[c] = c < limit ? ds[c] : 0.0f;
                }
                float sum[2] = {0.0f, 0.0f};
#pragma unroll
                for (int c = 0; c < 32; c += 2) add2(sum[0], sum[1], sum[0], sum[1], ds[c], ds[c + 1]);
                drift += sum[0] + sum[1];
            }
#pragma unroll
            for (int c = 0; c < 16; ++c) out[c] = pack2<T>(ds[2 * c], ds[2 * c + 1]);
            tmem_st16(s_at, out);                                     // over the first half of what this thread read
            wait_st();
            fence_before();
            __syncwarp();
            if (lane == 0) barrier_arrive(bar(qDs));
        }
        const float row_drift = single ? 0.0f : over_parts(drift);
        // A row of one key has P = 1 and dS = 0 whatever its score: what the recomputed P leaves of dS is rounding and nothing
        // else.  (Times 0: a NaN stays one.)
        float factor = seen == 1 ? 0.0f : p.scale;
        if (ok) ok = wait(qDone, 0);
        if (stopped(sync)) ok = false;                                // (qDone comes in any case)
        if (!ok) factor = NAN;                                        // given up: dQ and, through delta, dK say so
        fence_after();
        T *row = static_cast<T *>(p.dq.p) + (live ? row_of(w, p.dq, w.head, i, w.q_first) : 0);
        // (a row past the sequence's end may hold anything: its probabilities are 0, and 0 is what they multiply)
        auto write_stat = [&](float off) {
            if (part < 2) stat_block(p, w, w.head, w.tile)[part * kTile + r] = part == 0 ? minus_lse : live ? minus_delta - off : 0.0f;
        };
        if (p.split == 1) {
            write_stat(ok ? row_drift : NAN);
            if (n > 0) {
                uint32_t o[DIM / 4];
                if constexpr (DIM == 128) tmem_ld32(tm_dq + my_lane + 32 * part, o);
                else tmem_ld16(tm_dq + my_lane + 16 * part, o);
                wait_ld(o);
                if (live) store_columns<T, DIM / 4>(row, part * (DIM / 4), p.dim, o, factor);
            } else if (live && part == 0) {
                zero_columns<T>(row, p.dim);
            }
        } else {
            // Every CTA lays its sums out in shared memory, [column][row] and the rows' drift; a share of the columns is added up
            // by each.  The first CTA, which has the first key tile, knows the row's delta.
            const uint32_t mine = base + r * 4, mine_drift = smem_address(row_delta + r);
            uint32_t o[DIM / 4];
            if constexpr (DIM == 128) tmem_ld32(tm_dq + my_lane + 32 * part, o);
            else tmem_ld16(tm_dq + my_lane + 16 * part, o);           // (what it holds does not matter where there was no key tile)
            wait_ld(o);
#pragma unroll
            for (int e = 0; e < DIM / 4; ++e)
                asm volatile("st.shared.u32 [%0], %1;" :: "r"(mine + (part * (DIM / 4) + e) * (kTile * 4)), "r"(!ok ? kNan : n > 0 ? o[e] : 0u) : "memory");
            if (part == 0) row_delta[r] = !ok ? NAN : n > 0 ? row_drift : 0.0f;
            cluster_sync();
            if (rank == 0) {
                float off = 0.0f;
                for (int k = 0; k < p.split; ++k) off += load_peer(mine_drift, k);
                write_stat(off);
            }
            const int share = DIM / p.split, each = share / 4 > 8 ? share / 4 : 8;   // columns of this CTA, and of a thread
            for (int col = rank * share + part * each; col < rank * share + min((part + 1) * each, share); col += 8) {
                float v[8] = {0.0f, 0.0f, 0.0f, 0.0f, 0.0f, 0.0f, 0.0f, 0.0f};
                for (int k = 0; k < p.split; ++k) {
                    float x[8];
#pragma unroll
                    for (int e = 0; e < 8; ++e) x[e] = load_peer(mine + (col + e) * (kTile * 4), k);
#pragma unroll
                    for (int e = 0; e < 8; ++e) v[e] += x[e];
                }
                uint32_t y[8];
#pragma unroll
                for (int e = 0; e < 8; ++e) y[e] = __float_as_uint(v[e]);
                if (live) store_columns<T, 8>(row, col, p.dim, y, factor);
            }
            cluster_sync();                                           // nobody's shared memory goes before it has been read
        }
    }
    end_cta(tmem);
}

// ---------------------------------------------------------------------------------------------------
// backward, dK and dV
// ---------------------------------------------------------------------------------------------------
// Four products (2048 clocks) and 1024 of exponentials for each row and key tile.  The key tile's K stays in tensor memory and
// its V in shared memory, so that Q and dO have three stages each.  What is left between the products is the chain of one
// tile: S, its exponentials, dP, dS, and their way through tensor memory, 2850 clocks with two tiles' products interleaved.
// Tensor pipe 60 % active on 4 x 2048 rows, 16 heads on 4, causal, where it takes half of the pass's 275 us.
// Barriers: v, k in tensor memory, q full/empty (3 stages), g full/empty (3 stages), statistics full/empty (2 stages), S full
// and read, dP full and read, P ready and used, dS ready and used, done.
enum { kV = 0, kK = 1, kQFull = 2, kQEmpty = 5, kGFull = 8, kGEmpty = 11, kTFull = 14, kTEmpty = 16, kS = 18, kSRead = 19, kDp = 20, kDpRead = 21, kP = 22,
       kPUsed = 23, kDs = 24, kDsUsed = 25, kDone = 26, kBars = 27 };

template <int DIM> constexpr int dkv_smem() { return 7 * (DIM / 64) * static_cast<int>(kHalfTile) + 2 * kStatBytes + static_cast<int>(sizeof(Sync)); }

template <typename T, int DIM>
__global__ void __launch_bounds__(kThreadsAttn, 1)
attention_dkv_kernel(const __grid_constant__ Params p) {
    constexpr int HALVES = DIM / 64;
    constexpr uint32_t kBytes = HALVES * kHalfTile;
    extern __shared__ __align__(1024) uint8_t raw[];
    const uint32_t base = smem_address(raw);
    float *stat = reinterpret_cast<float *>(raw + 7 * kBytes);        // [stage][-lse * log2 e, -delta][128]
    Sync *sync = reinterpret_cast<Sync *>(raw + 7 * kBytes + 2 * kStatBytes);
    const int warp = uniform(static_cast<int>(threadIdx.x >> 5)), lane = threadIdx.x & 31;
    // Behind the dQ kernel only the statistics are still to come (whatever ran before it has ended, or it would not have
    // started): they are waited for where they are loaded.  Every CTA waits, so that this grid never ends before that one.
    if (!p.after_dq) pdl_wait();
    const int rank = p.split > 1 ? static_cast<int>(cluster_rank()) : 0;
    const Work w = find_work(p, blockIdx.x / p.split, p.kv_heads, false);
    if (w.packed && w.batch == p.batch) {                             // (the whole cluster)
        if (rank == 0) {
            fill_outside<T>(p, w, p.k_offsets, p.k_rows, p.k_len, p.dk, nullptr);
            fill_outside<T>(p, w, p.k_offsets, p.k_rows, p.k_len, p.dv, nullptr);
        }
        pdl_wait();
        return;
    }
    const int k0 = w.tile * kTile;
    if (k0 >= w.k_len) {
        pdl_wait();
        return;
    }
    // row tiles [first, last) see a key of this tile; all query heads of the group, one after the other, dealt out to the
    // cluster's CTAs in turn
    const int reach = w.k_len - w.q_len;                              // row i sees keys up to i + reach
    const int first = p.causal ? max(0, k0 - reach) / kTile : 0;
    const int each = max(0, (w.q_len + kTile - 1) / kTile - first);
    const int n = uniform(share_of(each * p.group, rank, p.split));

    // a quarter of a row of the K tile for each thread, read while the CTA sets itself up
    uint32_t keys[DIM / 8];
    if (warp < kMmaWarp && n > 0) {
        const int i = k0 + (threadIdx.x & 127), first_col = (warp >> 2) * (DIM / 4);
        const T *src = static_cast<const T *>(p.kin.p) + (i < w.k_len ? row_of(w, p.kin, w.head, i, w.k_first) : 0);
#pragma unroll
        for (int c = 0; c < DIM / 4; c += 8) {
            const uint4 v = i < w.k_len && first_col + c < p.dim ? __ldg(reinterpret_cast<const uint4 *>(src + first_col + c)) : make_uint4(0, 0, 0, 0);
            keys[c / 2] = v.x; keys[c / 2 + 1] = v.y; keys[c / 2 + 2] = v.z; keys[c / 2 + 3] = v.w;
        }
    }

    constexpr uint32_t counts[kBars] = {1, 16, 1, 1, 1, 1, 1, 1, 1, 1, 1, 1, 1, 1, 1, 1, 16, 16, 1, 16, 1, 16, 16, 1, 16, 1, 1};
    const uint32_t tmem = start_cta(sync, kBars, counts);
    auto bar = [&](int i) { return smem_address(&sync->bar[i]); };
    auto wait = [&](int i, uint32_t parity) { return barrier_wait(bar(i), parity, &sync->stop, p.timeouts); };
    const uint32_t sm_v = base, sm_q = base + kBytes, sm_g = base + 4 * kBytes;
    // tensor memory: one place for S and dP in turn (each is read into registers at once, which frees it), one for P and dS in
    // turn, the K tile, dV, dK
    const uint32_t tm_s = tmem, tm_dp = tmem, tm_p = tmem + kTile, tm_ds = tm_p, tm_k = tm_p + kTile / 2, tm_dv = tmem + 2 * kTile, tm_dk = tmem + 3 * kTile;

    bool ok = true;
    if (warp >= kMmaWarp) {
        give_registers<kDkvIssue>();
        if (warp == kLoadWarp) {
            int issued_q = 0, issued_t = 0, issued_g = 0;
            if (n > 0 && lane == 0) {
                prefetch_map(&p.q);
                prefetch_map(&p.v);
                prefetch_map(&p.g);
                barrier_expect(bar(kV), kBytes);
                load_halves<HALVES>(sm_v, &p.v, w.k_first + k0, w.head, w.q_batch, bar(kV));
            }
            if (n == 0) pdl_wait();
            for (int j = 0; j < n; ++j) {
                const int s = j & 1, s3 = j % 3, at = rank + j * p.split;
                const int head = w.head * p.group + at / each, tile = first + at % each, q0 = tile * kTile;
                const uint32_t again = ((j >> 1) & 1) ^ 1;
                if (!wait(kQEmpty + s3, ((j / 3) & 1) ^ 1)) break;
                if (lane == 0) {
                    barrier_expect(bar(kQFull + s3), kBytes);
                    load_halves<HALVES>(sm_q + s3 * kBytes, &p.q, w.q_first + q0, head, w.q_batch, bar(kQFull + s3));
                }
                issued_q = j + 1;
                if (j == 0) pdl_wait();
                if (!wait(kTEmpty + s, again)) break;
                if (lane == 0) {
                    barrier_expect(bar(kTFull + s), kStatBytes);
                    load_bytes(smem_address(stat + s * 2 * kTile), stat_block(p, w, head, tile), kStatBytes, bar(kTFull + s));
                }
                issued_t = j + 1;
                if (!wait(kGEmpty + s3, ((j / 3) & 1) ^ 1)) break;
                if (lane == 0) {
                    barrier_expect(bar(kGFull + s3), kBytes);
                    load_halves<HALVES>(sm_g + s3 * kBytes, &p.g, w.q_first + q0, head, w.q_batch, bar(kGFull + s3));
                }
                issued_g = j + 1;
            }
            if (stopped(sync)) {
                if (n > 0) barrier_wait(bar(kV), 0, nullptr, p.timeouts);
                for (int s = 0; s < 3; ++s) {
                    if (issued_q > s) barrier_wait(bar(kQFull + s), ((issued_q - 1 - s) / 3) & 1, nullptr, p.timeouts);
                    if (issued_g > s) barrier_wait(bar(kGFull + s), ((issued_g - 1 - s) / 3) & 1, nullptr, p.timeouts);
                }
                for (int s = 0; s < 2; ++s)
                    if (issued_t > s) barrier_wait(bar(kTFull + s), ((issued_t - 1 - s) >> 1) & 1, nullptr, p.timeouts);
            }
        } else if (warp == kMmaWarp) {
            const uint32_t leader = elect_leader();
            // Q tile j is used by S_j and, transposed, by dK_j; G tile j by dP_j and, transposed, by dV_j
            auto rows_left = [&](int j) { return w.q_len - (first + (rank + j * p.split) % each) * kTile; };
            auto scores = [&](int j) {
                const uint32_t tile = sm_q + (j % 3) * kBytes;
                if (!wait(kQFull + j % 3, (j / 3) & 1)) return false;
                if (w.packed && rows_left(j) < kTile) clear_rows<HALVES>(tile, rows_left(j));
                product_rows_tmem<T, DIM>(leader, tm_s, tm_k, tile);
                commit(leader, bar(kS));
                return true;
            };
            auto dprobs = [&](int j) {
                const uint32_t tile = sm_g + (j % 3) * kBytes;
                if (!wait(kGFull + j % 3, (j / 3) & 1)) return false;
                if (w.packed && rows_left(j) < kTile) clear_rows<HALVES>(tile, rows_left(j));
                product_rows<T, DIM>(leader, tm_dp, sm_v, tile);
                commit(leader, bar(kDp));
                return true;
            };
            ok = n == 0 || wait(kK, 0);
            fence_after();
            ok = ok && (n == 0 || (scores(0) && wait(kV, 0) && wait(kSRead, 0)));
            fence_after();
            if (ok && n > 0) ok = dprobs(0);
            for (int j = 0; ok && j < n; ++j) {
                ok = wait(kP, j & 1);                                 // P_j written
                if (!ok) break;
                fence_after();
                product_columns<T, DIM, 8, 64>(leader, tm_dv, tm_p, sm_g + (j % 3) * kBytes, j > 0);
                commit(leader, bar(kPUsed));
                commit(leader, bar(kGEmpty + j % 3));
                ok = wait(kDpRead, j & 1);                            // dP_j is in registers: S_j+1 may take its place
                if (!ok) break;
                fence_after();
                if (j + 1 < n && !(ok = scores(j + 1))) break;
                ok = wait(kDs, j & 1);                                // dS_j written over P_j
                if (!ok) break;
                fence_after();
                product_columns<T, DIM, 8, 64>(leader, tm_dk, tm_ds, sm_q + (j % 3) * kBytes, j > 0);
                commit(leader, bar(kDsUsed));
                commit(leader, bar(kQEmpty + j % 3));
                if (j + 1 < n) {
                    ok = wait(kSRead, (j + 1) & 1);                   // S_j+1 is in registers: dP_j+1 may take its place
                    if (!ok) break;
                    fence_after();
                    ok = dprobs(j + 1);
                }
            }
            commit(leader, bar(kDone));
            barrier_wait(bar(kDone), 0, nullptr, p.timeouts);
        }
        if (p.split > 1) {                                            // the element-wise warps' two barriers, below
            cluster_sync();
            cluster_sync();
        }
    } else {
        take_registers<kDkvWork>();
        const int part = warp >> 2;                                   // rows [32 part, 32 part + 32) of every row tile
        const int row_key = k0 + (threadIdx.x & 127);                 // this thread's row of K, dV and dK
        const int key = k0 + 32 * (warp & 3) + lane / 4;              // the first of its 4 keys, 8 apart, in S and dP
        const uint32_t my_lane = static_cast<uint32_t>(warp & 3) << 21;
        if (n > 0) {                                                  // the K tile to tensor memory
            if constexpr (DIM == 128) tmem_st16(tm_k + 16 * part + my_lane, keys);
            else tmem_st8(tm_k + 8 * part + my_lane, keys);
            wait_st();
            fence_before();
            __syncwarp();
            if (lane == 0) barrier_arrive(bar(kK));
        }
        const int alone = p.causal && k0 == 0 && reach <= 0 ? -reach : INT_MIN;   // the one row that sees key 0 and no other
        int tile = rank;                                              // of this head, from `first` on
        for (int j = 0; j < n; ++j, tile += p.split) {
            while (tile >= each) tile -= each;                        // the next head
            const int q0 = (first + tile) * kTile;
            // A thread holds 8 rows' values for each of 4 keys, not 32 rows' for one: the statistics that it reads are a quarter.
            // They are read before the scores are there: afterwards dP's product, whose operands both lie in shared memory,
            // leaves other reads of it waiting.
            const float2 *l2 = reinterpret_cast<const float2 *>(stat + (j & 1) * 2 * kTile + 32 * part) + lane % 4;
            const float2 *d2 = l2 + kTile / 2;
            ok = wait(kTFull + (j & 1), (j >> 1) & 1);
            if (!ok) break;
            const float2 minus_lse[4] = {l2[0], l2[4], l2[8], l2[12]};
            ok = wait(kS, j & 1);
            if (!ok) break;
            fence_after();
            uint32_t s[32], out[16];
            float prob[32];
            tmem_ld_16x32(tm_s + 32 * part + my_lane, s);
            tmem_ld_16x32(tm_s + 32 * part + my_lane + (16u << 16), s + 16);
            wait_ld(s);
            fence_before();
            __syncwarp();
            if (lane == 0) barrier_arrive(bar(kSRead));
            // rows past the end and rows that see nothing have -lse = -inf: their probabilities are 0
            if (p.causal && k0 + kTile - 1 > q0 + reach) {            // some rows do not see some keys
                const int from = key - reach - q0 - 32 * part - 2 * (lane % 4);   // of the first of the 4 keys, which are 8 apart
#pragma unroll
                for (int c = 0; c < 4; ++c) {
                    const float2 l = minus_lse[c];
#pragma unroll
                    for (int k = 0; k < 4; ++k) {
                        const int x = 16 * (k / 2) + 4 * c + 2 * (k % 2);
                        exp2_scaled<false>(prob[x], prob[x + 1], __uint_as_float(s[x]), __uint_as_float(s[x + 1]), p.scale_log2, l.x, l.y);
                        prob[x] = 8 * c >= from + 8 * k ? prob[x] : 0.0f;
                        prob[x + 1] = 8 * c + 1 >= from + 8 * k ? prob[x + 1] : 0.0f;
                    }
                }
            } else {
#pragma unroll
                for (int c = 0; c < 4; ++c) {
                    const float2 l = minus_lse[c];
#pragma unroll
                    for (int k = 0; k < 4; ++k) {
                        const int x = 16 * (k / 2) + 4 * c + 2 * (k % 2);
                        if (k == 3) exp2_scaled<true>(prob[x], prob[x + 1], __uint_as_float(s[x]), __uint_as_float(s[x + 1]), p.scale_log2, l.x, l.y);
                        else exp2_scaled<false>(prob[x], prob[x + 1], __uint_as_float(s[x]), __uint_as_float(s[x + 1]), p.scale_log2, l.x, l.y);
                    }
                }
            }
#pragma unroll
            for (int c = 0; c < 16; ++c) out[c] = pack2<T>(prob[2 * c], prob[2 * c + 1]);
            ok = j == 0 || wait(kDsUsed, (j - 1) & 1);
            if (!ok) break;
            fence_after();
            tmem_st_16x16(tm_p + 16 * part + my_lane, out);
            tmem_st_16x16(tm_p + 16 * part + my_lane + (16u << 16), out + 8);
            wait_st();
            fence_before();
            __syncwarp();
            if (lane == 0) barrier_arrive(bar(kP));
            if (static_cast<uint32_t>(alone - q0) < kTile) {          // its P is 1 and its dS 0, as in the dQ kernel
                const int place = alone - q0 - 32 * part - 2 * (lane % 4);
#pragma unroll
                for (int x = 0; x < 32; ++x)
                    if (8 * (x / 4 % 4) + x % 2 == place) prob[x] = 0.0f;
            }
            ok = wait(kDp, j & 1);
            if (!ok) break;
            fence_after();
#pragma unroll
            for (int h = 0; h < 2; ++h) {                             // 16 keys at a time
                uint32_t d[16];
                tmem_ld_16x32(tm_dp + 32 * part + my_lane + (static_cast<uint32_t>(16 * h) << 16), d);
                wait_ld(d);
#pragma unroll
                for (int c = 0; c < 4; ++c) {
                    const float2 e = d2[4 * c];
#pragma unroll
                    for (int k = 0; k < 2; ++k) {
                        const int x = 4 * c + 2 * k;
                        float v0, v1;
                        add2(v0, v1, __uint_as_float(d[x]), __uint_as_float(d[x + 1]), e.x, e.y);
                        mul2(v0, v1, v0, v1, prob[16 * h + x], prob[16 * h + x + 1]);
                        out[8 * h + x / 2] = pack2<T>(v0, v1);
                    }
                }
            }
            fence_before();
            __syncwarp();
            if (lane == 0) barrier_arrive(bar(kDpRead));
            ok = wait(kPUsed, j & 1);
            if (!ok) break;
            fence_after();
            tmem_st_16x16(tm_ds + 16 * part + my_lane, out);
            tmem_st_16x16(tm_ds + 16 * part + my_lane + (16u << 16), out + 8);
            wait_st();
            fence_before();
            __syncwarp();
            if (lane == 0) {
                barrier_arrive(bar(kDs));
                barrier_arrive(bar(kTEmpty + (j & 1)));
            }
        }
        if (ok) ok = wait(kDone, 0);
        if (stopped(sync)) ok = false;                                // (kDone comes in any case)
        fence_after();
        // dV by every other four warps, dK by the rest; the first eight warps take the first half of the columns
        const int which = part & 1, half = part >> 1, r = threadIdx.x & 127;
        const bool live = row_key < w.k_len;
        const Rows &to = which == 0 ? p.dv : p.dk;
        // (rows of one key have no dS; NaN: a wait was given up)
        const float factor = !ok ? NAN : which == 0 ? 1.0f : w.k_len == 1 ? 0.0f : p.scale;
        const uint32_t from = (which == 0 ? tm_dv : tm_dk) + my_lane;
        T *row = static_cast<T *>(to.p) + (live ? row_of(w, to, w.head, row_key, w.k_first) : 0);
        if (p.split == 1) {
            if (n > 0) {
#pragma unroll
                for (int c = 0; c < DIM / 64; ++c) {
                    uint32_t o[32];
                    const int col = half * (DIM / 2) + 32 * c;
                    tmem_ld32(from + col, o);
                    wait_ld(o);
                    if (live) store_columns<T, 32>(row, col, p.dim, o, factor);
                }
            } else if (live && half == 0) {
                zero_columns<T>(row, p.dim);
            }
        } else {
            // Each CTA adds up a share of the columns over the cluster, and lays the others of its sums out in its own shared
            // memory, [dV or dK][column][key] (the tiles are no longer needed), for their CTAs.
            const uint32_t mine = base + static_cast<uint32_t>(which * DIM) * (kTile * 4) + r * 4;
            const int share = DIM / p.split;
#pragma unroll
            for (int c = 0; c < DIM / 64; ++c) {
                uint32_t o[32];
                const int col = half * (DIM / 2) + 32 * c;
                if (share >= 32 && col / share == rank) continue;
                tmem_ld32(from + col, o);                             // (what it holds does not matter where there was no row tile)
                wait_ld(o);
#pragma unroll
                for (int e = 0; e < 32; ++e)
                    asm volatile("st.shared.u32 [%0], %1;" :: "r"(mine + (col + e) * (kTile * 4)), "r"(!ok ? kNan : n > 0 ? o[e] : 0u) : "memory");
            }
            cluster_sync();
            auto add_up = [&](auto columns) {                         // this thread's columns of the share: half of them
                constexpr int N = decltype(columns)::value;
                uint32_t o[N];
                const int col = rank * share + half * N;
                if constexpr (N == 32) tmem_ld32(from + col, o);
                else if constexpr (N == 16) tmem_ld16(from + col, o);
                else tmem_ld8(from + col, o);
                wait_ld(o);
                for (int k = 1; k < p.split; ++k) {
                    const uint32_t peer = static_cast<uint32_t>((rank + k) % p.split);
                    float v[N];
#pragma unroll
                    for (int e = 0; e < N; ++e) v[e] = load_peer(mine + (col + e) * (kTile * 4), peer);
#pragma unroll
                    for (int e = 0; e < N; ++e) o[e] = __float_as_uint((k == 1 && n == 0 ? 0.0f : __uint_as_float(o[e])) + v[e]);
                }
                cluster_arrive();                                     // nobody's shared memory goes before it has been read
                if (live) store_columns<T, N>(row, col, p.dim, o, factor);
            };
            if (share / 2 == 32) add_up(std::integral_constant<int, 32>{});
            else if (share / 2 == 16) add_up(std::integral_constant<int, 16>{});
            else add_up(std::integral_constant<int, 8>{});
            cluster_wait();
        }
    }
    end_cta(tmem);
}

}  // namespace attn
}  // namespace fewbit
