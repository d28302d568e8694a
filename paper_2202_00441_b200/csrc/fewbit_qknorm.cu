// RMS norm of every query and key head with the position rotation in the same pass, and its gradients
// (fewbit_qk_norm_rope_fwd / _bwd).
//
// Mathematics, for one head x of D elements with weight w and the rotation R of its token's position:
//   r = rsqrt(mean(x^2) + eps),  y = R (x r w)
//   g' = R^T g,  dw = sum over heads of g' x r,  dx = r (g' w - x r^2 mean(g' w x))
// Memory bound: 2 (forward) or 3 (backward) elements moved for each element, some 10 to 30 operations.
//
// Decomposition: a head belongs to G lanes (a power of two).  A lane holds a "unit": two pieces of V
// elements that the rotation pairs with one another ((j, j + rotary_dim/2) pairs: pieces rotary_dim/2
// apart; neighbouring pairs: pieces side by side), so no value ever changes lanes and the sums are a
// few shuffles.  A group works on kHeads heads of ONE token at a time: the token's cosines and sines are
// read once for all of them, and their loads are in flight together.
#include <cmath>

#include "fewbit_device.cuh"

namespace fewbit {
bool pdl_enabled();
int device_sm_count(cudaError_t *err);

namespace {

constexpr int kQkThreads = 256;
constexpr int kQkMaxDim = 256;
constexpr int kFwdHeads = 4, kBwdHeads = 2;
constexpr int kBwdCtasPerSm = 2;

struct QkTensor {
    void *p;
    long long b, i, h;                  // strides in elements
};
struct QkParams {
    QkTensor in[2], g[2], out[2];       // [query, key]; g: incoming gradients (backward)
    const float *weight[2];
    const float *cos, *sin;
    const void *positions;
    float *partial;                     // backward: (CTAs, 2, head_dim) sums of the weights' gradients, or nullptr
    long long table_rows;
    uint32_t tokens, length;
    int heads[2];
    int jobs[2];                        // head groups of one token: queries, keys
    int dim, rot, half;                 // half = rot / 2
    int units, rot_units;               // units of a head; those that are rotated half against half
    int group;                          // G
    bool interleaved, positions64;
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

__device__ __forceinline__ float group_sum(float x, int group) {
    for (int o = group >> 1; o > 0; o >>= 1) x += __shfl_xor_sync(0xffffffffu, x, o);
    return x;
}

// Where a lane's units lie, and the rotation of their pairs for one position.
template <int V, int CU>
struct Units {
    int a[CU], b[CU];                   // first element of each piece; b < 0: no second piece, a < 0: no unit
    __device__ __forceinline__ void place(const QkParams &q, int sub) {
#pragma unroll
        for (int c = 0; c < CU; ++c) {
            const int u = sub + c * q.group;
            a[c] = b[c] = -1;
            if (u >= q.units) continue;
            if (u < q.rot_units) {
                a[c] = u * V;
                b[c] = q.half + u * V;
            } else {
                a[c] = 2 * q.rot_units * V + 2 * (u - q.rot_units) * V;
                b[c] = a[c] + V < q.dim ? a[c] + V : -1;
            }
        }
    }
};

// cos and sin of a lane's pairs at one position: for units rotated half against half, V pairs; for neighbouring
// pairs, V/2 pairs of each piece (with V = 1 the unit's two pieces are the pair).  Pairs that are not rotated get (1, 0).
template <int V, int CU>
struct Turn {
    float c[CU][V], s[CU][V];
    __device__ __forceinline__ void load(const QkParams &q, const Units<V, CU> &u, long long pos) {
        const bool known = pos >= 0 && pos < q.table_rows;
        const float bad = __uint_as_float(0x7fc00000u);
        const long long row = known ? pos * q.half : 0;
#pragma unroll
        for (int k = 0; k < CU; ++k)
#pragma unroll
            for (int e = 0; e < V; ++e) {
                int j = -1;                                   // the pair's column of the tables
                if (u.a[k] >= 0) {
                    if (!q.interleaved) j = u.a[k] + V <= q.half ? u.a[k] + e : -1;
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
    // (va, vb) <- R (va, vb), or R^T when `back`
    __device__ __forceinline__ void apply(const QkParams &q, float (&va)[CU][V], float (&vb)[CU][V], bool back) const {
#pragma unroll
        for (int k = 0; k < CU; ++k) {
            if (!q.interleaved || V == 1) {
#pragma unroll
                for (int e = 0; e < V; ++e) {
                    const float sn = back ? -s[k][e] : s[k][e];
                    const float x = va[k][e], y = vb[k][e];
                    va[k][e] = x * c[k][e] - y * sn;
                    vb[k][e] = x * sn + y * c[k][e];
                }
            } else {
#pragma unroll
                for (int e = 0; e < V; ++e) {
                    const float sn = back ? -s[k][e] : s[k][e];
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

template <typename T, int V, int CU, int NH>
__device__ __forceinline__ void load_heads(const T *base, long long step, int n, const Units<V, CU> &u, Chunk<T, V> (&x)[NH][CU][2]) {
#pragma unroll
    for (int j = 0; j < NH; ++j)
#pragma unroll
        for (int c = 0; c < CU; ++c) {
            x[j][c][0].zero();
            x[j][c][1].zero();
            if (j < n) {
                if (u.a[c] >= 0) x[j][c][0].load(base + j * step + u.a[c]);
                if (u.b[c] >= 0) x[j][c][1].load(base + j * step + u.b[c]);
            }
        }
}

template <typename T, int V, int CU>
__device__ __forceinline__ void store_head(T *base, const Units<V, CU> &u, const float (&va)[CU][V], const float (&vb)[CU][V]) {
#pragma unroll
    for (int c = 0; c < CU; ++c) {
        if (u.a[c] >= 0) store_chunk<T, V>(base + u.a[c], va[c]);
        if (u.b[c] >= 0) store_chunk<T, V>(base + u.b[c], vb[c]);
    }
}

template <int V, int CU>
__device__ __forceinline__ void load_weight(const float *w, const Units<V, CU> &u, float (&wa)[CU][V], float (&wb)[CU][V]) {
#pragma unroll
    for (int c = 0; c < CU; ++c)
#pragma unroll
        for (int e = 0; e < V; ++e) {
            wa[c][e] = w == nullptr ? 1.0f : (u.a[c] >= 0 ? __ldg(w + u.a[c] + e) : 0.0f);
            wb[c][e] = w == nullptr ? 1.0f : (u.b[c] >= 0 ? __ldg(w + u.b[c] + e) : 0.0f);
        }
}

template <typename T, int V, int CU>
__global__ void __launch_bounds__(kQkThreads)
qk_fwd_kernel(const __grid_constant__ QkParams q) {
    pdl_launch_dependents();
    const int sub = threadIdx.x & (q.group - 1);
    const uint32_t per = kQkThreads / q.group;                      // groups of a CTA
    const uint32_t jobs = q.jobs[0] + q.jobs[1];
    const uint32_t total = q.tokens * jobs;                         // < 2^31 by the host's check
    Units<V, CU> u;
    u.place(q, sub);
    pdl_wait();
    // every lane of a warp runs the same number of rounds (the sums' shuffles need them all)
    for (uint32_t base = blockIdx.x * per; base < total; base += gridDim.x * per) {
        const uint32_t job = base + threadIdx.x / q.group;
        const bool live = job < total;
        const uint32_t token = live ? job / jobs : 0, part = live ? job % jobs : 0;
        const int which = part >= static_cast<uint32_t>(q.jobs[0]);
        const int head = (part - (which ? q.jobs[0] : 0)) * kFwdHeads;
        const int n = live ? min(kFwdHeads, q.heads[which] - head) : 0;
        const uint32_t bi = token / q.length, i = token % q.length;
        const QkTensor &in = q.in[which], &out = q.out[which];
        const T *src = static_cast<const T *>(in.p) + bi * in.b + i * in.i + head * in.h;
        Chunk<T, V> x[kFwdHeads][CU][2];
        load_heads<T, V, CU, kFwdHeads>(src, in.h, n, u, x);
        Turn<V, CU> turn;
        turn.load(q, u, position_of(q, token, i));
        float wa[CU][V], wb[CU][V];
        load_weight<V, CU>(q.weight[which], u, wa, wb);
        T *dst = static_cast<T *>(out.p) + bi * out.b + i * out.i + head * out.h;
#pragma unroll
        for (int j = 0; j < kFwdHeads; ++j) {
            float va[CU][V], vb[CU][V], sum = 0.0f;
#pragma unroll
            for (int c = 0; c < CU; ++c) {
                x[j][c][0].widen(va[c]);
                x[j][c][1].widen(vb[c]);
#pragma unroll
                for (int e = 0; e < V; ++e) sum += va[c][e] * va[c][e] + vb[c][e] * vb[c][e];
            }
            const float r = rsqrtf(group_sum(sum, q.group) * q.inv_dim + q.eps);
            if (j >= n) continue;
#pragma unroll
            for (int c = 0; c < CU; ++c)
#pragma unroll
                for (int e = 0; e < V; ++e) { va[c][e] *= r * wa[c][e]; vb[c][e] *= r * wb[c][e]; }
            turn.apply(q, va, vb, false);
            store_head<T, V, CU>(dst + j * out.h, u, va, vb);
        }
    }
}

template <typename T, int V, int CU>
__global__ void __launch_bounds__(kQkThreads)
qk_bwd_kernel(const __grid_constant__ QkParams q) {
    pdl_launch_dependents();
    const int sub = threadIdx.x & (q.group - 1);
    const uint32_t per = kQkThreads / q.group;
    Units<V, CU> u;
    u.place(q, sub);
    __shared__ float sums[kQkThreads / 32][2 * V * CU][33];
    pdl_wait();
#pragma unroll 1
    for (int which = 0; which < 2; ++which) {                       // queries, then keys: one set of weight sums at a time
        const uint32_t jobs = q.jobs[which];
        const uint32_t total = q.tokens * jobs;
        float wa[CU][V], wb[CU][V], da[CU][V], db[CU][V];
        load_weight<V, CU>(q.weight[which], u, wa, wb);
#pragma unroll
        for (int c = 0; c < CU; ++c)
#pragma unroll
            for (int e = 0; e < V; ++e) da[c][e] = db[c][e] = 0.0f;
        const QkTensor &in = q.in[which], &gin = q.g[which], &out = q.out[which];
        for (uint32_t base = blockIdx.x * per; base < total; base += gridDim.x * per) {
            const uint32_t job = base + threadIdx.x / q.group;
            const bool live = job < total;
            const uint32_t token = live ? job / jobs : 0;
            const int head = live ? (job % jobs) * kBwdHeads : 0;
            const int n = live ? min(kBwdHeads, q.heads[which] - head) : 0;
            const uint32_t bi = token / q.length, i = token % q.length;
            Chunk<T, V> x[kBwdHeads][CU][2], g[kBwdHeads][CU][2];
            load_heads<T, V, CU, kBwdHeads>(static_cast<const T *>(in.p) + bi * in.b + i * in.i + head * in.h, in.h, n, u, x);
            load_heads<T, V, CU, kBwdHeads>(static_cast<const T *>(gin.p) + bi * gin.b + i * gin.i + head * gin.h, gin.h, n, u, g);
            Turn<V, CU> turn;
            turn.load(q, u, position_of(q, token, i));
            T *dst = static_cast<T *>(out.p) + bi * out.b + i * out.i + head * out.h;
#pragma unroll
            for (int j = 0; j < kBwdHeads; ++j) {
                float va[CU][V], vb[CU][V], ga[CU][V], gb[CU][V], sum = 0.0f, dot = 0.0f;
#pragma unroll
                for (int c = 0; c < CU; ++c) {
                    x[j][c][0].widen(va[c]);
                    x[j][c][1].widen(vb[c]);
                    g[j][c][0].widen(ga[c]);
                    g[j][c][1].widen(gb[c]);
                }
                turn.apply(q, ga, gb, true);
#pragma unroll
                for (int c = 0; c < CU; ++c)
#pragma unroll
                    for (int e = 0; e < V; ++e) {
                        sum += va[c][e] * va[c][e] + vb[c][e] * vb[c][e];
                        dot += ga[c][e] * wa[c][e] * va[c][e] + gb[c][e] * wb[c][e] * vb[c][e];
                    }
                const float r = rsqrtf(group_sum(sum, q.group) * q.inv_dim + q.eps);
                const float shift = group_sum(dot, q.group) * q.inv_dim * r * r;
                if (j >= n) continue;
#pragma unroll
                for (int c = 0; c < CU; ++c)
#pragma unroll
                    for (int e = 0; e < V; ++e) {
                        da[c][e] += ga[c][e] * (va[c][e] * r);
                        db[c][e] += gb[c][e] * (vb[c][e] * r);
                        va[c][e] = r * (ga[c][e] * wa[c][e] - va[c][e] * shift);
                        vb[c][e] = r * (gb[c][e] * wb[c][e] - vb[c][e] * shift);
                    }
                store_head<T, V, CU>(dst + j * out.h, u, va, vb);
            }
        }
        if (q.partial == nullptr) continue;
        // the CTA's sum of every element of the weight, in a fixed order: lane by lane through shared memory
        __syncthreads();
#pragma unroll
        for (int c = 0; c < CU; ++c)
#pragma unroll
            for (int e = 0; e < V; ++e) {
                sums[threadIdx.x >> 5][(2 * c) * V + e][threadIdx.x & 31] = da[c][e];
                sums[threadIdx.x >> 5][(2 * c + 1) * V + e][threadIdx.x & 31] = db[c][e];
            }
        __syncthreads();
        if (threadIdx.x < static_cast<unsigned>(q.group)) {
            float *row = q.partial + (static_cast<size_t>(blockIdx.x) * 2 + which) * q.dim;
#pragma unroll
            for (int c = 0; c < CU; ++c)
#pragma unroll
                for (int e = 0; e < 2 * V; ++e) {
                    const int first = e < V ? u.a[c] : u.b[c];
                    if (first < 0) continue;
                    float total_sum = 0.0f;
                    for (int w = 0; w < kQkThreads / 32; ++w)
                        for (int l = sub; l < 32; l += q.group) total_sum += sums[w][2 * c * V + e][l];
                    row[first + e % V] = total_sum;
                }
        }
    }
}

// Adds up the CTAs' partial sums: 32 columns and 32 rows of threads for each CTA.
__global__ void __launch_bounds__(1024)
qk_weight_kernel(const float *partial, int ctas, int dim, float *dq, float *dk) {
    pdl_launch_dependents();
    __shared__ float part[32][33];
    const int lane = threadIdx.x & 31, row = threadIdx.x >> 5;
    const int col = blockIdx.x * 32 + lane;                          // of 2 * dim
    pdl_wait();
    float sum = 0.0f;
    if (col < 2 * dim)
        for (int c = row; c < ctas; c += 32) sum += partial[static_cast<size_t>(c) * 2 * dim + col];
    part[row][lane] = sum;
    __syncthreads();
    if (row == 0 && col < 2 * dim) {
        sum = 0.0f;
        for (int r = 0; r < 32; ++r) sum += part[r][lane];
        float *to = col < dim ? dq : dk;
        if (to != nullptr) to[col < dim ? col : col - dim] = sum;
    }
}

using QkLaunch = cudaError_t (*)(const QkParams &, unsigned, cudaStream_t);
template <typename T, int V, int CU>
cudaError_t launch_fwd(const QkParams &q, unsigned grid, cudaStream_t st) {
    return launch_pdl(qk_fwd_kernel<T, V, CU>, grid, kQkThreads, 0, st, pdl_enabled(), q);
}
template <typename T, int V, int CU>
cudaError_t launch_bwd_qk(const QkParams &q, unsigned grid, cudaStream_t st) {
    return launch_pdl(qk_bwd_kernel<T, V, CU>, grid, kQkThreads, 0, st, pdl_enabled(), q);
}
// [dtype][log2 V]; a lane holds CU units so that 32 lanes cover the largest head
const QkLaunch kQkFwd[3][4] = {
    {launch_fwd<float, 1, 4>, launch_fwd<float, 2, 2>, launch_fwd<float, 4, 1>, nullptr},
    {launch_fwd<__nv_bfloat16, 1, 4>, launch_fwd<__nv_bfloat16, 2, 2>, launch_fwd<__nv_bfloat16, 4, 1>, launch_fwd<__nv_bfloat16, 8, 1>},
    {launch_fwd<__half, 1, 4>, launch_fwd<__half, 2, 2>, launch_fwd<__half, 4, 1>, launch_fwd<__half, 8, 1>},
};
const QkLaunch kQkBwd[3][4] = {
    {launch_bwd_qk<float, 1, 4>, launch_bwd_qk<float, 2, 2>, launch_bwd_qk<float, 4, 1>, nullptr},
    {launch_bwd_qk<__nv_bfloat16, 1, 4>, launch_bwd_qk<__nv_bfloat16, 2, 2>, launch_bwd_qk<__nv_bfloat16, 4, 1>, launch_bwd_qk<__nv_bfloat16, 8, 1>},
    {launch_bwd_qk<__half, 1, 4>, launch_bwd_qk<__half, 2, 2>, launch_bwd_qk<__half, 4, 1>, launch_bwd_qk<__half, 8, 1>},
};

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
        if (s->heads > 1 << 20 || s->kv_heads > 1 << 20 || s->batch > most / s->length ||
            s->batch * s->length > most / (static_cast<int64_t>(s->heads) + s->kv_heads + 1))
            return FEWBIT_ERR_TOO_LARGE;
    }
    auto bad = [](const void *p, uintptr_t a) { return (reinterpret_cast<uintptr_t>(p) & (a - 1)) != 0; };
    if (bad(s->cos, 4) || bad(s->sin, 4) || bad(s->q_weight, 4) || bad(s->k_weight, 4) || bad(s->positions, s->positions_are_64bit ? 8 : 4))
        return FEWBIT_ERR_ALIGNMENT;
    return FEWBIT_OK;
}

// Fills what both directions share; `all` are the tensors of the call (n of them, query and key in turn).
fewbit_status fill(const fewbit_qk_shape *s, const fewbit_heads *const *all, int n, int heads_per_job, QkParams *q, int *log_v) {
    const int elem = s->dtype == FEWBIT_F32 ? 4 : 2;
    int v = 16 / elem;
    auto halve = [&](uint64_t bits) { while (v > 1 && bits % v != 0) v >>= 1; };
    halve(s->head_dim);
    if (!s->interleaved) halve(s->rotary_dim / 2);
    for (int k = 0; k < n; ++k) {
        if ((k % 2 ? s->kv_heads : s->heads) == 0) continue;
        const fewbit_heads *t = all[k];
        if (t == nullptr || t->data == nullptr) return FEWBIT_ERR_INVALID_ARG;
        const uintptr_t at = reinterpret_cast<uintptr_t>(t->data);
        if (at % elem) return FEWBIT_ERR_ALIGNMENT;
        halve(at / elem);
        if (s->batch > 1) halve(static_cast<uint64_t>(t->batch_stride));
        if (s->length > 1) halve(static_cast<uint64_t>(t->row_stride));
        if ((k % 2 ? s->kv_heads : s->heads) > 1) halve(static_cast<uint64_t>(t->head_stride));
    }
    *log_v = v == 8 ? 3 : v == 4 ? 2 : v == 2 ? 1 : 0;
    q->weight[0] = s->q_weight;
    q->weight[1] = s->k_weight;
    q->cos = s->cos;
    q->sin = s->sin;
    q->positions = s->rotary_dim > 0 ? s->positions : nullptr;
    q->table_rows = s->rotary_dim > 0 ? s->table_rows : INT64_MAX;
    q->partial = nullptr;
    q->tokens = static_cast<uint32_t>(s->batch * s->length);
    q->length = static_cast<uint32_t>(s->length > 0 ? s->length : 1);
    q->heads[0] = s->heads;
    q->heads[1] = s->kv_heads;
    for (int k = 0; k < 2; ++k) q->jobs[k] = (q->heads[k] + heads_per_job - 1) / heads_per_job;
    q->dim = s->head_dim;
    q->rot = s->rotary_dim;
    q->half = s->rotary_dim / 2;
    q->interleaved = s->interleaved != 0;
    q->rot_units = s->interleaved ? 0 : q->half / v;
    q->units = q->rot_units + (s->head_dim - 2 * q->rot_units * v + 2 * v - 1) / (2 * v);
    q->group = 1;
    while (q->group < q->units && q->group < 32) q->group *= 2;
    q->positions64 = s->positions_are_64bit != 0;
    q->eps = s->eps;
    q->inv_dim = 1.0f / static_cast<float>(s->head_dim);
    return FEWBIT_OK;
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
    QkParams q;
    int log_v = 0;
    const fewbit_heads *all[4] = {qi, ki, qo, ko};
    if (const fewbit_status st = fill(s, all, 4, kFwdHeads, &q, &log_v); st != FEWBIT_OK) return st;
    q.in[0] = tensor(qi); q.in[1] = tensor(ki);
    q.out[0] = tensor(qo); q.out[1] = tensor(ko);
    cudaError_t err = cudaSuccess;
    const unsigned sms = device_sm_count(&err);
    if (err != cudaSuccess) return cuda_status(err);
    const uint64_t groups = static_cast<uint64_t>(q.tokens) * (q.jobs[0] + q.jobs[1]);
    const uint64_t per = kQkThreads / q.group, want = (groups + per - 1) / per, most = static_cast<uint64_t>(sms) * 16;
    err = kQkFwd[s->dtype][log_v](q, static_cast<unsigned>(want < most ? want : most), static_cast<cudaStream_t>(stream));
    if (err == cudaSuccess) g_launches.fetch_add(1, std::memory_order_relaxed);
    return cuda_status(err);
}

size_t fewbit_qk_norm_rope_workspace_bytes(const fewbit_qk_shape *s) {
    using namespace fewbit;
    if (check_shape(s) != FEWBIT_OK) return 0;
    cudaError_t err = cudaSuccess;
    const unsigned sms = device_sm_count(&err);
    return err != cudaSuccess ? 0 : static_cast<size_t>(sms) * kBwdCtasPerSm * 2 * s->head_dim * sizeof(float);
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
    QkParams q;
    int log_v = 0;
    const fewbit_heads *all[6] = {gqo, gko, qi, ki, gq, gk};
    if (const fewbit_status st = fill(s, all, 6, kBwdHeads, &q, &log_v); st != FEWBIT_OK) return st;
    if (weights && workspace == nullptr) return FEWBIT_ERR_INVALID_ARG;
    if (weights && (at & 15)) return FEWBIT_ERR_ALIGNMENT;
    q.g[0] = tensor(gqo); q.g[1] = tensor(gko);
    q.in[0] = tensor(qi); q.in[1] = tensor(ki);
    q.out[0] = tensor(gq); q.out[1] = tensor(gk);
    cudaError_t err = cudaSuccess;
    const unsigned sms = device_sm_count(&err);
    if (err != cudaSuccess) return cuda_status(err);
    const uint64_t per = kQkThreads / q.group, groups = static_cast<uint64_t>(q.tokens) * (q.jobs[0] > q.jobs[1] ? q.jobs[0] : q.jobs[1]);
    const uint64_t want = (groups + per - 1) / per, most = static_cast<uint64_t>(sms) * kBwdCtasPerSm;
    const unsigned grid = static_cast<unsigned>(want < most ? want : most);
    if (weights && workspace_bytes < static_cast<size_t>(grid) * 2 * s->head_dim * sizeof(float)) return FEWBIT_ERR_ALLOC;
    if (weights) q.partial = static_cast<float *>(workspace);
    err = kQkBwd[s->dtype][log_v](q, grid, stm);
    if (err != cudaSuccess) return cuda_status(err);
    g_launches.fetch_add(1, std::memory_order_relaxed);
    if (!weights) return FEWBIT_OK;
    err = launch_pdl(qk_weight_kernel, (2 * s->head_dim + 31) / 32, 1024, 0, stm, pdl_enabled(), q.partial, static_cast<int>(grid), s->head_dim, dqw, dkw);
    if (err == cudaSuccess) g_launches.fetch_add(1, std::memory_order_relaxed);
    return cuda_status(err);
}

}  // extern "C"
