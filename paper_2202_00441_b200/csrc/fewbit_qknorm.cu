// RMS norm of every query and key head with the position rotation in the same pass, and its gradients
// (fewbit_qk_norm_rope_fwd / _bwd).
//
// Mathematics, for one head x of D elements with weight w and the rotation R of its token's position:
//   r = rsqrt(mean(x^2) + eps),  y = R (x r w)
//   g' = R^T g,  dw = sum over heads of g' x r,  dx = r (g' w - x r^2 mean(g' w x))
// Memory bound: 2 (forward) or 3 (backward) elements moved for each element, some 10 to 30 operations.
//
// Decomposition: a head belongs to G lanes (a power of two).  A lane holds a "unit": two pieces of V
// elements, where those of the one are rotated with those of the other (pairs (j, j + rotary_dim/2)) or each holds whole
// pairs (neighbouring ones), so no value ever changes lanes and the sums are a few shuffles; neighbouring lanes'
// pieces are neighbours.  A CTA works on one chunk of heads (blockIdx.y) for a stride of tokens: a group reads a
// token's cosines and sines once for the chunk, and some heads are in flight at a time.
#include <atomic>
#include <cmath>

#include "fewbit_device.cuh"
#include "fewbit_packed.cuh"

namespace fewbit {
bool pdl_enabled();
int device_sm_count(cudaError_t *err);

namespace {

constexpr int kQkThreads = 256;
constexpr int kQkMaxDim = 256;
// Heads in flight and CTAs on an SM, chosen together: bytes in flight against registers.  Measured on 4 x 8192 tokens,
// 32 + 8 heads of 128, bfloat16, forward / backward in us, back to back on the same tensors: (4, 2 CTAs) 111 / -, (4, 3) 129 / -, (2, 3) 137 / -, (2, 4) 143 / -;
// (2, 2) - / 210, (1, 2) - / 213, (1, 3) - / 306, (2, 3) - / 361 (spilled registers).  With copies ahead (Ahead, below) the
// backward pass takes 162 to 168, and 176 = 88 % of the copy bandwidth where every pass has other tensors than the last (back to
// back, part of what the last pass wrote is still in L2); heads half of which are rotated 245 -> 165, neighbouring pairs 284 -> 172, heads of 96 elements 233 -> 148, of 80 227 -> 147.  The forward
// pass of 16-bit types, 116 = 89 % with other tensors each time, loses by them with full lanes (1, 2, 3, 5 heads ahead: 147, 121, 131, 133; bursts of
// 4 or 8 heads: 132, 126): its bursts of loads between stores suit the memory better.  Binary32 gains with 2 heads ahead,
// 235 -> 215 (3: 236; 222 = 92 % with other tensors each time), and so do the forms without full lanes (2 / 3 heads ahead): heads half of which are rotated
// 135 -> 113 / 119, of 96 elements 128 -> 103 / 96, of 80 121 -> 97 / 93.
constexpr int kFwdHeads = 4, kBwdHeads = 2;
constexpr int kChunkHeads = 8;
constexpr int kFwdCtasPerSm = 2, kBwdCtasPerSm = 2;

struct QkTensor {
    void *p;
    long long b, i, h;                  // strides in elements
};
struct QkParams {
    QkTensor in[2], g[2], out[2];       // [query, key]; g: incoming gradients (backward)
    const float *weight[2];
    const float *cos, *sin;
    const void *positions;
    float *partial;                     // backward: a row of head_dim sums of the weight's gradient for each CTA, or nullptr
    long long table_rows;
    uint32_t tokens, length;
    int heads[2];
    int chunks[2], chunk;               // chunks of `chunk` heads: queries, keys
    int dim, rot, half;                 // half = rot / 2
    int units, rot_units;               // units of a head; those that are rotated half against half
    int group;                          // G
    bool positions64, vector_tables;    // vector_tables: 16-byte reads of four columns of cos and sin are aligned
    float eps, inv_dim;
};

template <int BYTES> struct Piece;
template <> struct Piece<16> { using type = uint4; };
template <> struct Piece<8> { using type = uint2; };
template <> struct Piece<4> { using type = uint32_t; };
template <> struct Piece<2> { using type = uint16_t; };

template <typename T, int V>
struct Chunk {
    using Raw = typename Piece<V * sizeof(T)>::type;
    Raw raw;
    __device__ __forceinline__ void load(const T *p) { raw = *reinterpret_cast<const Raw *>(p); }
    __device__ __forceinline__ void zero() { raw = Raw{}; }
    __device__ __forceinline__ void widen(float (&v)[V]) const {
        T t[V];
        memcpy(t, &raw, sizeof(raw));
#pragma unroll
        for (int e = 0; e < V; ++e) v[e] = load1(&t[e]);
    }
};
template <typename T, int V>
__device__ __forceinline__ void store_chunk(T *p, const float (&v)[V]) {
    using Raw = typename Piece<V * sizeof(T)>::type;
    T t[V];
#pragma unroll
    for (int e = 0; e < V; ++e) store1(&t[e], v[e]);
    Raw raw;
    memcpy(&raw, t, sizeof(raw));
    *reinterpret_cast<Raw *>(p) = raw;
}

// d = a b, d = a b + c, over V elements; `scale` forms: b the same for all
template <int V> __device__ __forceinline__ void vmul(float (&d)[V], const float (&a)[V], const float (&b)[V]) {
    if constexpr (V == 1) d[0] = a[0] * b[0];
    else {
#pragma unroll
        for (int e = 0; e < V; e += 2) mul2(d[e], d[e + 1], a[e], a[e + 1], b[e], b[e + 1]);
    }
}
template <int V> __device__ __forceinline__ void vfma(float (&d)[V], const float (&a)[V], const float (&b)[V], const float (&c)[V]) {
    if constexpr (V == 1) d[0] = fmaf(a[0], b[0], c[0]);
    else {
#pragma unroll
        for (int e = 0; e < V; e += 2) fma2(d[e], d[e + 1], a[e], a[e + 1], b[e], b[e + 1], c[e], c[e + 1]);
    }
}
template <int V> __device__ __forceinline__ void vscale(float (&d)[V], const float (&a)[V], float b) {
    if constexpr (V == 1) d[0] = a[0] * b;
    else {
#pragma unroll
        for (int e = 0; e < V; e += 2) mul2(d[e], d[e + 1], a[e], a[e + 1], b, b);
    }
}
template <int V> __device__ __forceinline__ void vaxpy(float (&d)[V], const float (&a)[V], float b, const float (&c)[V]) {
    if constexpr (V == 1) d[0] = fmaf(a[0], b, c[0]);
    else {
#pragma unroll
        for (int e = 0; e < V; e += 2) fma2(d[e], d[e + 1], a[e], a[e + 1], b, b, c[e], c[e + 1]);
    }
}
// s += a b, in two running sums
template <int V> __device__ __forceinline__ void vdot(float (&s)[2], const float (&a)[V], const float (&b)[V]) {
    if constexpr (V == 1) s[0] = fmaf(a[0], b[0], s[0]);
    else {
#pragma unroll
        for (int e = 0; e < V; e += 2) fma2(s[0], s[1], a[e], a[e + 1], b[e], b[e + 1], s[0], s[1]);
    }
}

__device__ __forceinline__ float group_sum(float x, int group) {
    for (int o = group >> 1; o > 0; o >>= 1) x += __shfl_xor_sync(0xffffffffu, x, o);
    return x;
}

// Where a lane's units lie.  FULL: every lane has both pieces of each unit, and all of them are rotated.
template <int V, int CU, bool FULL>
struct Units {
    int a[CU], b[CU];                   // first element of each piece; b < 0: no second piece, a < 0: no unit
    __device__ __forceinline__ void place(const QkParams &q, int sub, bool interleaved) {
#pragma unroll
        for (int c = 0; c < CU; ++c) {
            const int u = sub + c * q.group;
            if (FULL) {
                a[c] = u * V;
                b[c] = q.half + a[c];
                continue;
            }
            a[c] = b[c] = -1;
            if (u >= q.units) continue;
            if (u < q.rot_units) {
                a[c] = u * V;
                b[c] = q.half + u * V;
            } else {
                const bool pairs = V == 1 && interleaved;             // single elements: a pair
                const int first = 2 * q.rot_units * V + (u - q.rot_units) * V;
                a[c] = pairs ? 2 * u : first;
                b[c] = pairs ? a[c] + 1 : first + (q.units - q.rot_units) * V;
                if (b[c] >= q.dim) b[c] = -1;
            }
        }
    }
    __device__ __forceinline__ bool has_a(int c) const { return FULL || a[c] >= 0; }
    __device__ __forceinline__ bool has_b(int c) const { return FULL || b[c] >= 0; }
};

// cos and sin of a lane's pairs at one position: for units rotated half against half, V pairs; for neighbouring
// pairs, V/2 pairs of each piece (with V = 1 the unit's two pieces are the pair).  Pairs that are not rotated get (1, 0).
template <int V, int CU, bool INTER, bool FULL>
struct Turn {
    float c[CU][V], s[CU][V];
    __device__ __forceinline__ void load(const QkParams &q, const Units<V, CU, FULL> &u, long long pos) {
        const bool known = pos >= 0 && pos < q.table_rows;
        const float bad = __uint_as_float(0x7fc00000u);
        const long long row = known ? pos * q.half : 0;
#pragma unroll
        for (int k = 0; k < CU; ++k) {
            if constexpr (V % 4 == 0) {
                // Columns in one run, or (neighbouring pairs) one for each piece; each rotated as a whole, or not at all.
                constexpr int RUNS = INTER ? 2 : 1, W = V / RUNS;
                bool none[RUNS], vectors = FULL || q.vector_tables;
#pragma unroll
                for (int h = 0; h < RUNS; ++h) {
                    const int at = h ? u.b[k] : u.a[k], end = INTER ? 2 * q.half : q.half;
                    none[h] = !FULL && (at < 0 || at >= end);
                    vectors = vectors && (FULL || none[h] || at + V <= end);
                }
                if (vectors) {
#pragma unroll
                    for (int h = 0; h < RUNS; ++h) {
                        const long long from = row + (INTER ? (h ? u.b[k] : u.a[k]) / 2 : u.a[k]);
#pragma unroll
                        for (int e = 0; e < W; ++e) {
                            c[k][h * W + e] = none[h] && known ? 1.0f : bad;
                            s[k][h * W + e] = 0.0f;
                        }
                        if (known && !none[h]) {
                            read<W>(&c[k][h * W], q.cos + from);
                            read<W>(&s[k][h * W], q.sin + from);
                        }
                    }
                    continue;
                }
            }
            if constexpr (!FULL) {
#pragma unroll
                for (int e = 0; e < V; ++e) {
                    int j = -1;                               // the pair's column of the tables
                    if (u.a[k] >= 0) {
                        if (!INTER) j = u.a[k] + V <= q.half ? u.a[k] + e : -1;
                        else if (V == 1) j = u.a[k] < q.rot ? u.a[k] / 2 : -1;
                        else {
                            const int first = e < V / 2 ? u.a[k] + 2 * e : u.b[k] + 2 * (e - V / 2);
                            j = (e < V / 2 || u.b[k] >= 0) && first < q.rot ? first / 2 : -1;
                        }
                    }
                    c[k][e] = !known ? bad : (j >= 0 ? __ldg(q.cos + row + j) : 1.0f);
                    s[k][e] = known && j >= 0 ? __ldg(q.sin + row + j) : 0.0f;
                }
            }
        }
    }
    template <int W>
    static __device__ __forceinline__ void read(float *to, const float *from) {
        if constexpr (W == 2) {
            const float2 x = __ldg(reinterpret_cast<const float2 *>(from));
            to[0] = x.x; to[1] = x.y;
        } else {
#pragma unroll
            for (int e = 0; e < W; e += 4) {
                const float4 x = __ldg(reinterpret_cast<const float4 *>(from + e));
                to[e] = x.x; to[e + 1] = x.y; to[e + 2] = x.z; to[e + 3] = x.w;
            }
        }
    }
    // (va, vb) <- R (va, vb), or R^T when BACK
    template <bool BACK>
    __device__ __forceinline__ void apply(float (&va)[CU][V], float (&vb)[CU][V]) const {
#pragma unroll
        for (int k = 0; k < CU; ++k) {
            if constexpr (!INTER || V == 1) {                 // a pair's elements lie in different pieces
                float to_a[V], to_b[V], x[V], y[V];
#pragma unroll
                for (int e = 0; e < V; ++e) {
                    to_a[e] = BACK ? s[k][e] : -s[k][e];
                    to_b[e] = -to_a[e];
                }
                vmul<V>(x, vb[k], to_a);
                vmul<V>(y, va[k], to_b);
                vfma<V>(va[k], va[k], c[k], x);
                vfma<V>(vb[k], vb[k], c[k], y);
            } else {
#pragma unroll
                for (int e = 0; e < V; ++e) {
                    const float sn = BACK ? -s[k][e] : s[k][e];
                    float &x = e < V / 2 ? va[k][2 * e % V] : vb[k][2 * e % V];
                    float &y = e < V / 2 ? va[k][(2 * e + 1) % V] : vb[k][(2 * e + 1) % V];
                    const float x0 = x, y0 = y;
                    x = x0 * c[k][e] - y0 * sn;
                    y = x0 * sn + y0 * c[k][e];
                }
            }
        }
    }
};

__device__ __forceinline__ long long position_of(const QkParams &q, uint32_t token, uint32_t i) {
    if (q.positions == nullptr) return i;
    return q.positions64 ? static_cast<const long long *>(q.positions)[token] : static_cast<const int *>(q.positions)[token];
}

template <typename T, int V, int CU, bool FULL>
__device__ __forceinline__ void load_head(const T *base, bool live, const Units<V, CU, FULL> &u, Chunk<T, V> (&x)[CU][2]) {
#pragma unroll
    for (int c = 0; c < CU; ++c) {
        x[c][0].zero();
        x[c][1].zero();
        if (live && u.has_a(c)) x[c][0].load(base + u.a[c]);
        if (live && u.has_b(c)) x[c][1].load(base + u.b[c]);
    }
}

template <typename T, int V, int CU, bool FULL>
__device__ __forceinline__ void store_head(T *base, const Units<V, CU, FULL> &u, const float (&va)[CU][V], const float (&vb)[CU][V]) {
#pragma unroll
    for (int c = 0; c < CU; ++c) {
        if (u.has_a(c)) store_chunk<T, V>(base + u.a[c], va[c]);
        if (u.has_b(c)) store_chunk<T, V>(base + u.b[c], vb[c]);
    }
}

template <int V, int CU, bool FULL>
__device__ __forceinline__ void load_weight(const float *w, const Units<V, CU, FULL> &u, float (&wa)[CU][V], float (&wb)[CU][V]) {
#pragma unroll
    for (int c = 0; c < CU; ++c)
#pragma unroll
        for (int e = 0; e < V; ++e) {
            wa[c][e] = w == nullptr ? 1.0f : (u.has_a(c) ? __ldg(w + u.a[c] + e) : 0.0f);
            wb[c][e] = w == nullptr ? 1.0f : (u.has_b(c) ? __ldg(w + u.b[c] + e) : 0.0f);
        }
}

// The chunk of heads [first, end) of queries (which = 0) or keys that a CTA works on.
struct HeadChunk {
    int which, first, end;
    __device__ __forceinline__ explicit HeadChunk(const QkParams &q) {
        which = static_cast<int>(blockIdx.y) >= q.chunks[0];
        first = (static_cast<int>(blockIdx.y) - (which ? q.chunks[0] : 0)) * q.chunk;
        end = min(first + q.chunk, q.heads[which]);
    }
};

// One head of the forward pass; `live`: it exists (all lanes take part in the sum).
template <typename T, int V, int CU, bool INTER, bool FULL>
__device__ __forceinline__ void fwd_head(const QkParams &q, const Units<V, CU, FULL> &u, const Turn<V, CU, INTER, FULL> &turn, const Chunk<T, V> (&x)[CU][2],
                                         const float (&wa)[CU][V], const float (&wb)[CU][V], bool live, T *dst) {
    float va[CU][V], vb[CU][V], sum[2] = {0.0f, 0.0f};
#pragma unroll
    for (int c = 0; c < CU; ++c) {
        x[c][0].widen(va[c]);
        x[c][1].widen(vb[c]);
        vdot<V>(sum, va[c], va[c]);
        vdot<V>(sum, vb[c], vb[c]);
    }
    const float r = rsqrtf(group_sum(sum[0] + sum[1], q.group) * q.inv_dim + q.eps);
    if (!live) return;
#pragma unroll
    for (int c = 0; c < CU; ++c) {
        vscale<V>(va[c], va[c], r);
        vscale<V>(vb[c], vb[c], r);
        vmul<V>(va[c], va[c], wa[c]);
        vmul<V>(vb[c], vb[c], wb[c]);
    }
    turn.template apply<false>(va, vb);
    store_head<T, V, CU, FULL>(dst, u, va, vb);
}

template <typename T, int V, int CU, bool INTER, bool FULL>
__global__ void __launch_bounds__(kQkThreads, kFwdCtasPerSm)
qk_fwd_kernel(const __grid_constant__ QkParams q) {
    pdl_launch_dependents();
    const uint32_t per = kQkThreads / q.group;                      // groups of a CTA
    const HeadChunk hc(q);
    const QkTensor &in = q.in[hc.which], &out = q.out[hc.which];
    Units<V, CU, FULL> u;
    u.place(q, threadIdx.x & (q.group - 1), INTER);
    pdl_wait();
    float wa[CU][V], wb[CU][V];
    load_weight<V, CU, FULL>(q.weight[hc.which], u, wa, wb);
    // every lane of a warp runs the same number of rounds (the sums' shuffles need them all)
    for (uint32_t base = blockIdx.x * per; base < q.tokens; base += gridDim.x * per) {
        const uint32_t token = base + threadIdx.x / q.group;
        const bool live = token < q.tokens;
        const uint32_t bi = live ? token / q.length : 0, i = live ? token % q.length : 0;
        Turn<V, CU, INTER, FULL> turn;
        turn.load(q, u, position_of(q, live ? token : 0, i));
        const T *src = static_cast<const T *>(in.p) + bi * in.b + i * in.i + hc.first * in.h;
        T *dst = static_cast<T *>(out.p) + bi * out.b + i * out.i + hc.first * out.h;
        for (int head = hc.first; head < hc.end; head += kFwdHeads, src += kFwdHeads * in.h, dst += kFwdHeads * out.h) {
            Chunk<T, V> x[kFwdHeads][CU][2];
#pragma unroll
            for (int j = 0; j < kFwdHeads; ++j) load_head<T, V, CU, FULL>(src + j * in.h, live && head + j < hc.end, u, x[j]);
#pragma unroll
            for (int j = 0; j < kFwdHeads; ++j) {
                fwd_head<T, V, CU, INTER, FULL>(q, u, turn, x[j], wa, wb, live && head + j < hc.end, dst + j * out.h);
            }
        }
    }
}

template <int V, int CU, bool FULL>
__device__ __forceinline__ void write_partial(const QkParams &q, const Units<V, CU, FULL> &u, float (&da)[CU][V], float (&db)[CU][V]) {
    if (q.partial == nullptr) return;
    __shared__ float sums[kQkThreads / 32][kQkMaxDim];
    // the CTA's sum of every element of the weight, in a fixed order: over a warp's groups, then over its warps
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
#pragma unroll
    for (int c = 0; c < CU; ++c)
#pragma unroll
        for (int e = 0; e < V; ++e) {
            for (int o = q.group; o < 32; o <<= 1) {
                da[c][e] += __shfl_xor_sync(0xffffffffu, da[c][e], o);
                db[c][e] += __shfl_xor_sync(0xffffffffu, db[c][e], o);
            }
            if (lane < q.group) {
                if (u.has_a(c)) sums[warp][u.a[c] + e] = da[c][e];
                if (u.has_b(c)) sums[warp][u.b[c] + e] = db[c][e];
            }
        }
    __syncthreads();
    if (static_cast<int>(threadIdx.x) < q.dim) {
        float total = 0.0f;
#pragma unroll
        for (int w = 0; w < kQkThreads / 32; ++w) total += sums[w][threadIdx.x];
        q.partial[(static_cast<size_t>(blockIdx.y) * gridDim.x + blockIdx.x) * q.dim + threadIdx.x] = total;
    }
}

// One head of the backward pass; `live`: it exists (all lanes take part in the sums).
template <typename T, int V, int CU, bool INTER, bool FULL>
__device__ __forceinline__ void bwd_head(const QkParams &q, const Units<V, CU, FULL> &u, const Turn<V, CU, INTER, FULL> &turn, const Chunk<T, V> (&x)[CU][2],
                                         const Chunk<T, V> (&g)[CU][2], const float (&wa)[CU][V], const float (&wb)[CU][V],
                                         float (&da)[CU][V], float (&db)[CU][V], bool live, T *dst) {
    float va[CU][V], vb[CU][V], ga[CU][V], gb[CU][V], squares[2] = {0.0f, 0.0f}, dots[2] = {0.0f, 0.0f};
#pragma unroll
    for (int c = 0; c < CU; ++c) {
        x[c][0].widen(va[c]);
        x[c][1].widen(vb[c]);
        g[c][0].widen(ga[c]);
        g[c][1].widen(gb[c]);
        vdot<V>(squares, va[c], va[c]);
        vdot<V>(squares, vb[c], vb[c]);
    }
    turn.template apply<true>(ga, gb);
    // t = g' x: the weight's gradient without r, and, times the weight, the terms of the dot product
    float ta[CU][V], tb[CU][V];
#pragma unroll
    for (int c = 0; c < CU; ++c) {
        vmul<V>(ta[c], ga[c], va[c]);
        vmul<V>(tb[c], gb[c], vb[c]);
        vdot<V>(dots, ta[c], wa[c]);
        vdot<V>(dots, tb[c], wb[c]);
    }
    float sum = squares[0] + squares[1], dot = dots[0] + dots[1];
    for (int o = q.group >> 1; o > 0; o >>= 1) {          // both sums in one go
        sum += __shfl_xor_sync(0xffffffffu, sum, o);
        dot += __shfl_xor_sync(0xffffffffu, dot, o);
    }
    const float r = rsqrtf(sum * q.inv_dim + q.eps);
    const float shift = -dot * q.inv_dim * r * r * r;
    if (!live) return;
#pragma unroll
    for (int c = 0; c < CU; ++c) {
        vaxpy<V>(da[c], ta[c], r, da[c]);
        vaxpy<V>(db[c], tb[c], r, db[c]);
        vscale<V>(ga[c], ga[c], r);                       // dx = (r g') w - (r^3 mean) x
        vscale<V>(gb[c], gb[c], r);
        vscale<V>(va[c], va[c], shift);
        vscale<V>(vb[c], vb[c], shift);
        vfma<V>(va[c], ga[c], wa[c], va[c]);
        vfma<V>(vb[c], gb[c], wb[c], vb[c]);
    }
    store_head<T, V, CU, FULL>(dst, u, va, vb);
}

template <typename T, int V, int CU, bool INTER, bool FULL>
__global__ void __launch_bounds__(kQkThreads, kBwdCtasPerSm)
qk_bwd_kernel(const __grid_constant__ QkParams q) {
    pdl_launch_dependents();
    const uint32_t per = kQkThreads / q.group;
    const HeadChunk hc(q);
    const QkTensor &in = q.in[hc.which], &gin = q.g[hc.which], &out = q.out[hc.which];
    Units<V, CU, FULL> u;
    u.place(q, threadIdx.x & (q.group - 1), INTER);
    pdl_wait();
    float wa[CU][V], wb[CU][V], da[CU][V], db[CU][V];
    load_weight<V, CU, FULL>(q.weight[hc.which], u, wa, wb);
#pragma unroll
    for (int c = 0; c < CU; ++c)
#pragma unroll
        for (int e = 0; e < V; ++e) da[c][e] = db[c][e] = 0.0f;
    for (uint32_t base = blockIdx.x * per; base < q.tokens; base += gridDim.x * per) {
        const uint32_t token = base + threadIdx.x / q.group;
        const bool live = token < q.tokens;
        const uint32_t bi = live ? token / q.length : 0, i = live ? token % q.length : 0;
        Turn<V, CU, INTER, FULL> turn;
        turn.load(q, u, position_of(q, live ? token : 0, i));
        const T *src = static_cast<const T *>(in.p) + bi * in.b + i * in.i + hc.first * in.h;
        const T *grd = static_cast<const T *>(gin.p) + bi * gin.b + i * gin.i + hc.first * gin.h;
        T *dst = static_cast<T *>(out.p) + bi * out.b + i * out.i + hc.first * out.h;
        for (int head = hc.first; head < hc.end; head += kBwdHeads, src += kBwdHeads * in.h, grd += kBwdHeads * gin.h, dst += kBwdHeads * out.h) {
            Chunk<T, V> x[kBwdHeads][CU][2], g[kBwdHeads][CU][2];
#pragma unroll
            for (int j = 0; j < kBwdHeads; ++j) {
                load_head<T, V, CU, FULL>(src + j * in.h, live && head + j < hc.end, u, x[j]);
                load_head<T, V, CU, FULL>(grd + j * gin.h, live && head + j < hc.end, u, g[j]);
            }
#pragma unroll
            for (int j = 0; j < kBwdHeads; ++j) {
                bwd_head<T, V, CU, INTER, FULL>(q, u, turn, x[j], g[j], wa, wb, da, db, live && head + j < hc.end, dst + j * out.h);
            }
        }
    }
    write_partial<V, CU, FULL>(q, u, da, db);
}

// What a thread will read of its heads is copied to shared memory ahead of its use, kAhead heads in advance and over the ends
// of tokens, so that loads are in flight all the time and take no registers.  No thread reads what another one copied.
// (Backward, more heads ahead suit the memory worse: 2, 3, 4, 5 heads 164, 188, 190, 191 us on the shape above, with tensors in one place,
// 178, 179, 179, 180 in another.)
template <int BYTES>
__device__ __forceinline__ void copy_ahead(uint32_t to, const void *from) {
    if constexpr (BYTES == 16) asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" :: "r"(to), "l"(from) : "memory");
    else asm volatile("cp.async.ca.shared.global [%0], [%1], 8;" :: "r"(to), "l"(from) : "memory");
}
template <typename T, int V, bool INTER, bool FULL, bool BACK>
struct Ahead {
    static constexpr int kAhead = BACK || FULL ? 2 : 3, kSlots = kAhead + 1;
    static constexpr int kItem = BACK ? 4 : 2, kBytes = V * sizeof(T);   // pieces of a head (values, gradients); bytes of each
    static constexpr uint32_t kPiece = kQkThreads * kBytes;
    static constexpr int kShared = kSlots * kItem * static_cast<int>(kPiece);
    uint32_t at;                                                      // this thread's place in a piece
    uint32_t base;                                                    // the next head to be copied: its token, ...
    int head = 0, heads;
    uint32_t slot = 0, used = 0;
    bool live = false;
    const T *x, *g;

    __device__ __forceinline__ uint32_t place(uint32_t slot, int k) const { return at + (slot * kItem + k) * kPiece; }
    __device__ __forceinline__ void start(const QkParams &q, const HeadChunk &hc, const Units<V, 1, FULL> &u, uint32_t shared) {
        at = shared + threadIdx.x * kBytes;
        base = blockIdx.x * (kQkThreads / q.group);
        heads = hc.end - hc.first;
        if constexpr (!FULL) {                                        // pieces that a lane does not have are zeros
            Chunk<T, V> none;
            none.zero();
#pragma unroll
            for (int k = 0; k < kSlots * kItem; ++k)
                if (!(k & 1 ? u.has_b(0) : u.has_a(0))) put(at + k * kPiece, none.raw);
        }
        for (int k = 0; k < kAhead; ++k) next(q, hc, u);
    }
    __device__ __forceinline__ void next(const QkParams &q, const HeadChunk &hc, const Units<V, 1, FULL> &u) {
        const QkTensor &xt = q.in[hc.which], &gt = q.g[hc.which];
        if (base < q.tokens) {
            if (head == 0) {
                const uint32_t token = base + threadIdx.x / q.group;
                live = token < q.tokens;
                if (live) {
                    const uint32_t bi = token / q.length, i = token % q.length;
                    x = static_cast<const T *>(xt.p) + bi * xt.b + i * xt.i + hc.first * xt.h;
                    if constexpr (BACK) g = static_cast<const T *>(gt.p) + bi * gt.b + i * gt.i + hc.first * gt.h;
                }
            }
            if (live) {
                if (u.has_a(0)) copy_ahead<kBytes>(place(slot, 0), x + u.a[0]);
                if (u.has_b(0)) copy_ahead<kBytes>(place(slot, 1), x + u.b[0]);
                x += xt.h;
                if constexpr (BACK) {
                    if (u.has_a(0)) copy_ahead<kBytes>(place(slot, 2), g + u.a[0]);
                    if (u.has_b(0)) copy_ahead<kBytes>(place(slot, 3), g + u.b[0]);
                    g += gt.h;
                }
            }
            slot = slot == kSlots - 1 ? 0 : slot + 1;
            if (++head == heads) {
                head = 0;
                base += gridDim.x * (kQkThreads / q.group);
            }
        }
        asm volatile("cp.async.commit_group;" ::: "memory");
    }
    static __device__ __forceinline__ void put(uint32_t to, uint4 r) {
        asm volatile("st.shared.v4.b32 [%0], {%1, %2, %3, %4};" :: "r"(to), "r"(r.x), "r"(r.y), "r"(r.z), "r"(r.w) : "memory");
    }
    static __device__ __forceinline__ void put(uint32_t to, uint2 r) {
        asm volatile("st.shared.v2.b32 [%0], {%1, %2};" :: "r"(to), "r"(r.x), "r"(r.y) : "memory");
    }
    static __device__ __forceinline__ void get(uint32_t from, uint4 &r) {
        asm volatile("ld.shared.v4.b32 {%0, %1, %2, %3}, [%4];" : "=r"(r.x), "=r"(r.y), "=r"(r.z), "=r"(r.w) : "r"(from) : "memory");
    }
    static __device__ __forceinline__ void get(uint32_t from, uint2 &r) {
        asm volatile("ld.shared.v2.b32 {%0, %1}, [%2];" : "=r"(r.x), "=r"(r.y) : "r"(from) : "memory");
    }
    // The oldest head: values, gradients
    __device__ __forceinline__ void take(Chunk<T, V> (&xs)[1][2], Chunk<T, V> (*gs)[2]) {
        asm volatile("cp.async.wait_group %0;" :: "n"(kAhead - 1) : "memory");
        get(place(used, 0), xs[0][0].raw);
        get(place(used, 1), xs[0][1].raw);
        if constexpr (BACK) {
            get(place(used, 2), gs[0][0].raw);
            get(place(used, 3), gs[0][1].raw);
        }
        used = used == kSlots - 1 ? 0 : used + 1;
    }
};

template <typename T, int V, bool INTER, bool FULL>
__global__ void __launch_bounds__(kQkThreads, kFwdCtasPerSm)
qk_fwd_ahead_kernel(const __grid_constant__ QkParams q) {
    extern __shared__ __align__(16) uint8_t shared[];
    pdl_launch_dependents();
    const HeadChunk hc(q);
    const QkTensor &out = q.out[hc.which];
    Units<V, 1, FULL> u;
    u.place(q, threadIdx.x & (q.group - 1), INTER);
    pdl_wait();
    Ahead<T, V, INTER, FULL, false> in;
    in.start(q, hc, u, static_cast<uint32_t>(__cvta_generic_to_shared(shared)));
    float wa[1][V], wb[1][V];
    load_weight<V, 1, FULL>(q.weight[hc.which], u, wa, wb);
    for (uint32_t base = blockIdx.x * (kQkThreads / q.group); base < q.tokens; base += gridDim.x * (kQkThreads / q.group)) {
        const uint32_t token = base + threadIdx.x / q.group;
        const bool live = token < q.tokens;
        const uint32_t bi = live ? token / q.length : 0, i = live ? token % q.length : 0;
        T *dst = static_cast<T *>(out.p) + bi * out.b + i * out.i + hc.first * out.h;
        Turn<V, 1, INTER, FULL> turn;
        turn.load(q, u, position_of(q, live ? token : 0, i));
        for (int head = hc.first; head < hc.end; ++head, dst += out.h) {
            Chunk<T, V> x[1][2];
            in.take(x, nullptr);
            in.next(q, hc, u);
            fwd_head<T, V, 1, INTER, FULL>(q, u, turn, x, wa, wb, live, dst);
        }
    }
}

template <typename T, int V, bool INTER, bool FULL>
__global__ void __launch_bounds__(kQkThreads, kBwdCtasPerSm)
qk_bwd_ahead_kernel(const __grid_constant__ QkParams q) {
    extern __shared__ __align__(16) uint8_t shared[];
    pdl_launch_dependents();
    const HeadChunk hc(q);
    const QkTensor &out = q.out[hc.which];
    Units<V, 1, FULL> u;
    u.place(q, threadIdx.x & (q.group - 1), INTER);
    pdl_wait();
    Ahead<T, V, INTER, FULL, true> in;
    in.start(q, hc, u, static_cast<uint32_t>(__cvta_generic_to_shared(shared)));
    float wa[1][V], wb[1][V], da[1][V], db[1][V];
    load_weight<V, 1, FULL>(q.weight[hc.which], u, wa, wb);
#pragma unroll
    for (int e = 0; e < V; ++e) da[0][e] = db[0][e] = 0.0f;
    for (uint32_t base = blockIdx.x * (kQkThreads / q.group); base < q.tokens; base += gridDim.x * (kQkThreads / q.group)) {
        const uint32_t token = base + threadIdx.x / q.group;
        const bool live = token < q.tokens;
        const uint32_t bi = live ? token / q.length : 0, i = live ? token % q.length : 0;
        T *dst = static_cast<T *>(out.p) + bi * out.b + i * out.i + hc.first * out.h;
        Turn<V, 1, INTER, FULL> turn;
        turn.load(q, u, position_of(q, live ? token : 0, i));
        for (int head = hc.first; head < hc.end; ++head, dst += out.h) {
            Chunk<T, V> x[1][2], g[1][2];
            in.take(x, g);
            in.next(q, hc, u);
            bwd_head<T, V, 1, INTER, FULL>(q, u, turn, x, g, wa, wb, da, db, live, dst);
        }
    }
    write_partial<V, 1, FULL>(q, u, da, db);
}

// Adds up the CTAs' partial sums, `q_ctas` rows of the queries' weight and then `k_ctas` of the keys': 32 columns and
// 32 rows of threads for each CTA (blockIdx.y: query or key).
__global__ void __launch_bounds__(1024)
qk_weight_kernel(const float *partial, int q_ctas, int k_ctas, int dim, float *dq, float *dk) {
    pdl_launch_dependents();
    __shared__ float part[32][33];
    const int lane = threadIdx.x & 31, row = threadIdx.x >> 5;
    const int col = blockIdx.x * 32 + lane;
    const int first = blockIdx.y ? q_ctas : 0, end = blockIdx.y ? q_ctas + k_ctas : q_ctas;
    pdl_wait();
    float sum = 0.0f;
    if (col < dim) {
#pragma unroll 8
        for (int c = first + row; c < end; c += 32) sum += partial[static_cast<size_t>(c) * dim + col];
    }
    part[row][lane] = sum;
    __syncthreads();
    sum = part[lane][row];                                           // transposed: a warp adds one column
    for (int o = 16; o > 0; o >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, o);
    float *to = blockIdx.y ? dk : dq;
    if (lane == 0 && blockIdx.x * 32 + row < dim && to != nullptr) to[blockIdx.x * 32 + row] = sum;
}

using QkLaunch = cudaError_t (*)(const QkParams &, unsigned, unsigned, cudaStream_t);
template <auto kernel, int smem>
cudaError_t launch_qk(const QkParams &q, unsigned x, unsigned y, cudaStream_t st) {
    if (smem > 0) {
        static std::atomic<unsigned long long> ready{0};              // devices (up to 64) whose limit has been raised
        int dev = 0;
        cudaError_t err = cudaGetDevice(&dev);
        if (err != cudaSuccess) return err;
        const unsigned long long bit = dev < 64 ? 1ull << dev : 0;
        if ((ready.load(std::memory_order_relaxed) & bit) == 0) {
            err = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, smem);
            if (err != cudaSuccess) return err;
            ready.fetch_or(bit, std::memory_order_relaxed);
        }
    }
    cudaLaunchConfig_t cfg = {};
    cfg.dynamicSmemBytes = smem;
    cfg.gridDim = dim3(x, y);
    cfg.blockDim = dim3(kQkThreads);
    cfg.stream = st;
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = attr;
    cfg.numAttrs = pdl_enabled() ? 1 : 0;
    return cudaLaunchKernelEx(&cfg, kernel, q);
}
template <typename T, int V, int CU, bool INTER, bool FULL>
cudaError_t launch_fwd(const QkParams &q, unsigned x, unsigned y, cudaStream_t st) {
    if constexpr (V > 1 && (!FULL || sizeof(T) == 4)) return launch_qk<qk_fwd_ahead_kernel<T, V, INTER, FULL>, Ahead<T, V, INTER, FULL, false>::kShared>(q, x, y, st);
    else return launch_qk<qk_fwd_kernel<T, V, CU, INTER, FULL>, 0>(q, x, y, st);
}
template <typename T, int V, int CU, bool INTER, bool FULL>
cudaError_t launch_bwd_qk(const QkParams &q, unsigned x, unsigned y, cudaStream_t st) {
    if constexpr (V > 1) return launch_qk<qk_bwd_ahead_kernel<T, V, INTER, FULL>, Ahead<T, V, INTER, FULL, true>::kShared>(q, x, y, st);
    else return launch_qk<qk_bwd_kernel<T, V, CU, INTER, FULL>, 0>(q, x, y, st);
}
// [dtype][interleaved][variant]: 16-byte pieces with full lanes, 16-byte pieces, 8-byte pieces of the 16-bit types, single
// elements; a lane holds CU units so that 32 lanes cover the largest head
enum { kFull, kWide, kHalfWide, kSingle, kVariants };
#define FEWBIT_QK_ROW(launch, T, V, INTER) \
    {launch<T, V, 1, INTER, true>, launch<T, V, 1, INTER, false>, launch<T, 4, 1, INTER, false>, launch<T, 1, 4, INTER, false>}
#define FEWBIT_QK_TABLE(launch) \
    {{FEWBIT_QK_ROW(launch, float, 4, false), FEWBIT_QK_ROW(launch, float, 4, true)}, \
     {FEWBIT_QK_ROW(launch, __nv_bfloat16, 8, false), FEWBIT_QK_ROW(launch, __nv_bfloat16, 8, true)}, \
     {FEWBIT_QK_ROW(launch, __half, 8, false), FEWBIT_QK_ROW(launch, __half, 8, true)}}
const QkLaunch kQkFwd[3][2][kVariants] = FEWBIT_QK_TABLE(launch_fwd);
const QkLaunch kQkBwd[3][2][kVariants] = FEWBIT_QK_TABLE(launch_bwd_qk);

fewbit_status check_shape(const fewbit_qk_shape *s) {
    if (s == nullptr || !valid_dtype(s->dtype) || s->batch < 0 || s->length < 0 || s->heads < 0 || s->kv_heads < 0 ||
        s->head_dim < 2 || s->head_dim % 2 || s->rotary_dim < 0 || s->rotary_dim % 2 || s->rotary_dim > s->head_dim ||
        !(s->eps >= 0) || !std::isfinite(s->eps))
        return FEWBIT_ERR_INVALID_ARG;
    if (s->head_dim > kQkMaxDim) return FEWBIT_ERR_UNSUPPORTED;
    if (s->rotary_dim > 0 && (s->cos == nullptr || s->sin == nullptr || s->table_rows < 0)) return FEWBIT_ERR_INVALID_ARG;
    if (s->rotary_dim > 0 && s->positions == nullptr && s->table_rows < s->length) return FEWBIT_ERR_INVALID_ARG;
    if (s->batch > 0 && s->length > 0) {
        const int64_t most = INT32_MAX;
        if (s->heads > 1 << 15 || s->kv_heads > 1 << 15 || s->batch > most / s->length ||
            s->batch * s->length > most / (static_cast<int64_t>(s->heads) + s->kv_heads + 1))
            return FEWBIT_ERR_TOO_LARGE;
    }
    auto bad = [](const void *p, uintptr_t a) { return (reinterpret_cast<uintptr_t>(p) & (a - 1)) != 0; };
    if (bad(s->cos, 4) || bad(s->sin, 4) || bad(s->q_weight, 4) || bad(s->k_weight, 4) || bad(s->positions, s->positions_are_64bit ? 8 : 4))
        return FEWBIT_ERR_ALIGNMENT;
    return FEWBIT_OK;
}

fewbit_status check_tensors(const fewbit_qk_shape *s, const fewbit_heads *const *all, int n) {
    for (int k = 0; k < n; ++k) {
        if ((k % 2 ? s->kv_heads : s->heads) == 0) continue;
        if (all[k] == nullptr || all[k]->data == nullptr) return FEWBIT_ERR_INVALID_ARG;
        if (reinterpret_cast<uintptr_t>(all[k]->data) % (s->dtype == FEWBIT_F32 ? 4 : 2)) return FEWBIT_ERR_ALIGNMENT;
    }
    return FEWBIT_OK;
}

// Fills what both directions share, and returns the kernels' variant; `all` are the tensors of the call (n of them, query
// and key in turn).
int fill(const fewbit_qk_shape *s, const fewbit_heads *const *all, int n, int heads_in_flight, unsigned sms, QkParams *q) {
    const int elem = s->dtype == FEWBIT_F32 ? 4 : 2;
    int v = 16 / elem;
    auto halve = [&](uint64_t bits) { while (v > 1 && bits % v != 0) v >>= 1; };
    halve(s->head_dim);
    if (!s->interleaved) halve(s->rotary_dim / 2);
    for (int k = 0; k < n; ++k) {
        if ((k % 2 ? s->kv_heads : s->heads) == 0) continue;
        const fewbit_heads *t = all[k];
        halve(reinterpret_cast<uintptr_t>(t->data) / elem);
        if (s->batch > 1) halve(static_cast<uint64_t>(t->batch_stride));
        if (s->length > 1) halve(static_cast<uint64_t>(t->row_stride));
        if ((k % 2 ? s->kv_heads : s->heads) > 1) halve(static_cast<uint64_t>(t->head_stride));
    }
    int variant = v == 16 / elem ? kWide : v >= 4 ? kHalfWide : kSingle;
    if (variant == kSingle) v = 1;
    q->weight[0] = s->q_weight;
    q->weight[1] = s->k_weight;
    q->cos = s->cos;
    q->sin = s->sin;
    q->positions = s->rotary_dim > 0 ? s->positions : nullptr;
    q->table_rows = s->rotary_dim > 0 ? s->table_rows : INT64_MAX;
    q->partial = nullptr;
    q->tokens = static_cast<uint32_t>(s->batch * s->length);
    q->length = static_cast<uint32_t>(s->length);
    q->heads[0] = s->heads;
    q->heads[1] = s->kv_heads;
    q->dim = s->head_dim;
    q->rot = s->rotary_dim;
    q->half = s->rotary_dim / 2;
    q->rot_units = s->interleaved ? 0 : q->half / v;
    q->units = q->rot_units + (s->head_dim - 2 * q->rot_units * v + 2 * v - 1) / (2 * v);
    q->group = 1;
    while (q->group < q->units && q->group < 32) q->group *= 2;
    const uintptr_t table = reinterpret_cast<uintptr_t>(s->cos) | reinterpret_cast<uintptr_t>(s->sin);
    if (variant == kWide && q->units == q->group && s->rotary_dim == s->head_dim && s->head_dim % (2 * v) == 0 && table % 16 == 0) variant = kFull;
    // whole chunks of heads amortise a token's cosines; a call too small to fill the SMs takes fewer heads at a time
    const uint32_t per = kQkThreads / q->group;
    for (q->chunk = kChunkHeads;; q->chunk /= 2) {
        for (int k = 0; k < 2; ++k) q->chunks[k] = (q->heads[k] + q->chunk - 1) / q->chunk;
        const uint64_t ctas = static_cast<uint64_t>((q->tokens + per - 1) / per) * (q->chunks[0] + q->chunks[1]);
        if (ctas >= sms || q->chunk <= heads_in_flight) break;
    }
    q->positions64 = s->positions_are_64bit != 0;
    q->vector_tables = table % 16 == 0 && q->half % 4 == 0;
    q->eps = s->eps;
    q->inv_dim = 1.0f / static_cast<float>(s->head_dim);
    return variant;
}

// CTAs along the tokens: all of them, or as many as keep `per_sm` CTAs on every SM busy
unsigned token_ctas(const QkParams &q, unsigned sms, int per_sm) {
    const unsigned per = kQkThreads / q.group, want = (q.tokens + per - 1) / per, rows = static_cast<unsigned>(q.chunks[0] + q.chunks[1]);
    const unsigned most = sms * per_sm / rows > 0 ? sms * per_sm / rows : 1;   // never a few CTAs more than fit at once
    return want < most ? want : most;
}

QkTensor tensor(const fewbit_heads *t) { return t == nullptr ? QkTensor{} : QkTensor{t->data, t->batch_stride, t->row_stride, t->head_stride}; }

fewbit_status cuda_status(cudaError_t err) {
    if (err == cudaSuccess) return FEWBIT_OK;
    t_last_cuda_error = static_cast<int>(err);
    return FEWBIT_ERR_CUDA;
}

}  // namespace
}  // namespace fewbit

extern "C" {

fewbit_status fewbit_qk_norm_rope_fwd(const fewbit_qk_shape *s, const fewbit_heads *qi, const fewbit_heads *ki, const fewbit_heads *qo,
                                      const fewbit_heads *ko, void *stream) {
    using namespace fewbit;
    if (const fewbit_status st = check_shape(s); st != FEWBIT_OK) return st;
    if (s->batch == 0 || s->length == 0 || s->heads + s->kv_heads == 0) return FEWBIT_OK;
    cudaError_t err = cudaSuccess;
    const fewbit_heads *all[4] = {qi, ki, qo, ko};
    if (const fewbit_status st = check_tensors(s, all, 4); st != FEWBIT_OK) return st;
    const unsigned sms = device_sm_count(&err);
    if (err != cudaSuccess) return cuda_status(err);
    QkParams q;
    const int variant = fill(s, all, 4, kFwdHeads, sms, &q);
    q.in[0] = tensor(qi); q.in[1] = tensor(ki);
    q.out[0] = tensor(qo); q.out[1] = tensor(ko);
    err = kQkFwd[s->dtype][s->interleaved != 0][variant](q, token_ctas(q, sms, kFwdCtasPerSm), q.chunks[0] + q.chunks[1], static_cast<cudaStream_t>(stream));
    if (err == cudaSuccess) g_launches.fetch_add(1, std::memory_order_relaxed);
    return cuda_status(err);
}

size_t fewbit_qk_norm_rope_workspace_bytes(const fewbit_qk_shape *s) {
    using namespace fewbit;
    if (check_shape(s) != FEWBIT_OK) return 0;
    cudaError_t err = cudaSuccess;
    const unsigned sms = device_sm_count(&err);
    // token_ctas rounds up once for each chunk of heads, of which there are at most this many
    const size_t chunks = static_cast<size_t>(s->heads + kBwdHeads - 1) / kBwdHeads + (s->kv_heads + kBwdHeads - 1) / kBwdHeads;
    return err != cudaSuccess ? 0 : (sms * kBwdCtasPerSm + chunks) * s->head_dim * sizeof(float);
}

fewbit_status fewbit_qk_norm_rope_bwd(const fewbit_qk_shape *s, const fewbit_heads *gqo, const fewbit_heads *gko, const fewbit_heads *qi,
                                      const fewbit_heads *ki, const fewbit_heads *gq, const fewbit_heads *gk, float *dqw, float *dkw,
                                      void *workspace, size_t workspace_bytes, void *stream) {
    using namespace fewbit;
    if (const fewbit_status st = check_shape(s); st != FEWBIT_OK) return st;
    const bool weights = dqw != nullptr || dkw != nullptr;
    const uintptr_t at = reinterpret_cast<uintptr_t>(workspace);
    if ((reinterpret_cast<uintptr_t>(dqw) | reinterpret_cast<uintptr_t>(dkw)) & 3) return FEWBIT_ERR_ALIGNMENT;
    const bool empty = s->batch == 0 || s->length == 0 || s->heads + s->kv_heads == 0;
    if (empty && !weights) return FEWBIT_OK;
    cudaStream_t stm = static_cast<cudaStream_t>(stream);
    if (empty) {                                             // the sums of nothing
        cudaError_t err = dqw ? cudaMemsetAsync(dqw, 0, s->head_dim * sizeof(float), stm) : cudaSuccess;
        if (err == cudaSuccess && dkw) err = cudaMemsetAsync(dkw, 0, s->head_dim * sizeof(float), stm);
        return cuda_status(err);
    }
    const fewbit_heads *all[6] = {gqo, gko, qi, ki, gq, gk};
    if (const fewbit_status st = check_tensors(s, all, 6); st != FEWBIT_OK) return st;
    if (weights && workspace == nullptr) return FEWBIT_ERR_INVALID_ARG;
    if (weights && (at & 15)) return FEWBIT_ERR_ALIGNMENT;
    cudaError_t err = cudaSuccess;
    const unsigned sms = device_sm_count(&err);
    if (err != cudaSuccess) return cuda_status(err);
    QkParams q;
    const int variant = fill(s, all, 6, kBwdHeads, sms, &q);
    q.g[0] = tensor(gqo); q.g[1] = tensor(gko);
    q.in[0] = tensor(qi); q.in[1] = tensor(ki);
    q.out[0] = tensor(gq); q.out[1] = tensor(gk);
    const unsigned x = token_ctas(q, sms, kBwdCtasPerSm), y = q.chunks[0] + q.chunks[1];
    if (weights && workspace_bytes < static_cast<size_t>(x) * y * s->head_dim * sizeof(float)) return FEWBIT_ERR_ALLOC;
    if (weights) q.partial = static_cast<float *>(workspace);
    err = kQkBwd[s->dtype][s->interleaved != 0][variant](q, x, y, stm);
    if (err != cudaSuccess) return cuda_status(err);
    g_launches.fetch_add(1, std::memory_order_relaxed);
    if (!weights) return FEWBIT_OK;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((s->head_dim + 31) / 32, 2);
    cfg.blockDim = dim3(1024);
    cfg.stream = stm;
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = attr;
    cfg.numAttrs = pdl_enabled() ? 1 : 0;
    err = cudaLaunchKernelEx(&cfg, qk_weight_kernel, static_cast<const float *>(q.partial), static_cast<int>(x) * q.chunks[0],
                             static_cast<int>(x) * q.chunks[1], s->head_dim, dqw, dkw);
    if (err == cudaSuccess) g_launches.fetch_add(1, std::memory_order_relaxed);
    return cuda_status(err);
}

}  // extern "C"
