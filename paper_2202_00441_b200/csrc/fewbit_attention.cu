// Entry points of attention: argument checks, tensor maps, launches.
#include "fewbit_attention.cuh"
#include "fewbit_attention_launch.h"

#include <cudaTypedefs.h>

#include <atomic>

namespace fewbit {
int device_sm_count(cudaError_t *err);

namespace {

using attn::Params;

__device__ unsigned int g_attention_timeouts;

fewbit_status cuda_status(cudaError_t err) {
    if (err == cudaSuccess) return FEWBIT_OK;
    t_last_cuda_error = static_cast<int>(err);
    return FEWBIT_ERR_CUDA;
}

PFN_cuTensorMapEncodeTiled_v12000 encode_function(cudaError_t *err) {
    static std::atomic<void *> cached{nullptr};
    void *fn = cached.load(std::memory_order_acquire);
    *err = cudaSuccess;
    if (fn == nullptr) {
        cudaDriverEntryPointQueryResult found;
        *err = cudaGetDriverEntryPointByVersion("cuTensorMapEncodeTiled", &fn, 12000, cudaEnableDefault, &found);
        if (*err == cudaSuccess && (found != cudaDriverEntryPointSuccess || fn == nullptr)) *err = cudaErrorNotSupported;
        if (*err != cudaSuccess) return nullptr;
        cached.store(fn, std::memory_order_release);
    }
    return reinterpret_cast<PFN_cuTensorMapEncodeTiled_v12000>(fn);
}

// Map of a (batch, rows, heads, dim) tensor as (dim, rows, heads, batch), read in boxes of 64 elements x 128 rows of one
// head; places past the tensor's rows or dim read as zero.
fewbit_status encode(CUtensorMap *map, const fewbit_heads *t, const fewbit_attention_shape *s, int64_t rows, int heads, int64_t batch) {
    cudaError_t err;
    const auto fn = encode_function(&err);
    if (fn == nullptr) return cuda_status(err);
    const cuuint64_t dense = static_cast<cuuint64_t>(s->head_dim) * 2;
    cuuint64_t dims[4] = {static_cast<cuuint64_t>(s->head_dim), static_cast<cuuint64_t>(rows), static_cast<cuuint64_t>(heads), static_cast<cuuint64_t>(batch)};
    // the stride of a dimension of length 1 is never used
    cuuint64_t strides[3] = {rows > 1 ? static_cast<cuuint64_t>(t->row_stride) * 2 : dense, heads > 1 ? static_cast<cuuint64_t>(t->head_stride) * 2 : dense,
                             batch > 1 ? static_cast<cuuint64_t>(t->batch_stride) * 2 : dense};
    cuuint32_t box[4] = {64, static_cast<cuuint32_t>(attn::kTile), 1, 1}, steps[4] = {1, 1, 1, 1};
    const CUresult r = fn(map, s->dtype == FEWBIT_F16 ? CU_TENSOR_MAP_DATA_TYPE_FLOAT16 : CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 4, t->data, dims, strides, box,
                          steps, CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
                          CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE);
    if (r != CUDA_SUCCESS) {
        t_last_cuda_error = static_cast<int>(r);
        return FEWBIT_ERR_CUDA;
    }
    return FEWBIT_OK;
}

struct Sizes {
    int64_t q_rows, k_rows;           // rows of the tensors
    int64_t batch;                    // of the tensors
    bool packed;
};

fewbit_status check_shape(const fewbit_attention_shape *s, Sizes *z) {
    if (s == nullptr || !valid_dtype(s->dtype) || s->batch < 0 || s->heads < 0 || s->kv_heads < 0 || s->head_dim < 1 || s->q_len < 0 || s->k_len < 0 ||
        !(s->scale > 0) || !std::isfinite(s->scale) || (s->q_offsets == nullptr) != (s->k_offsets == nullptr))
        return FEWBIT_ERR_INVALID_ARG;
    if (s->heads > 0 && (s->kv_heads == 0 || s->heads % s->kv_heads != 0)) return FEWBIT_ERR_INVALID_ARG;
    z->packed = s->q_offsets != nullptr;
    if (z->packed && (s->q_rows < 0 || s->k_rows < 0 || s->q_len > s->q_rows || s->k_len > s->k_rows)) return FEWBIT_ERR_INVALID_ARG;
    if (s->dtype == FEWBIT_F32 || s->head_dim % 8 != 0 || s->head_dim > 128) return FEWBIT_ERR_UNSUPPORTED;
    if ((reinterpret_cast<uintptr_t>(s->q_offsets) | reinterpret_cast<uintptr_t>(s->k_offsets)) & 3) return FEWBIT_ERR_ALIGNMENT;
    z->q_rows = z->packed ? s->q_rows : s->q_len;
    z->k_rows = z->packed ? s->k_rows : s->k_len;
    z->batch = z->packed ? 1 : s->batch;
    // tiles, heads and sequences are counted in 31 bits, rows too
    const int64_t most = INT32_MAX;
    const int64_t longest = s->q_len > s->k_len ? s->q_len : s->k_len;
    if (z->q_rows > most - 1024 || z->k_rows > most - 1024 ||
        (longest / attn::kTile + 1) > most / (static_cast<int64_t>(s->heads) + 1) / (static_cast<int64_t>(s->batch) + 1))
        return FEWBIT_ERR_TOO_LARGE;
    return FEWBIT_OK;
}

fewbit_status check_tensor(const fewbit_heads *t, int64_t rows, int heads, int64_t batch) {
    if (rows == 0 || heads == 0 || batch == 0) return FEWBIT_OK;
    if (t == nullptr || t->data == nullptr) return FEWBIT_ERR_INVALID_ARG;
    if (reinterpret_cast<uintptr_t>(t->data) & 15) return FEWBIT_ERR_ALIGNMENT;
    const int64_t strides[3] = {batch > 1 ? t->batch_stride : 8, rows > 1 ? t->row_stride : 8, heads > 1 ? t->head_stride : 8};
    for (int64_t x : strides) {
        if (x % 8 != 0) return FEWBIT_ERR_ALIGNMENT;
        if (x <= 0 || x >= (int64_t{1} << 39)) return FEWBIT_ERR_UNSUPPORTED;   // the tensor maps hold 40 bits of bytes, no sign
    }
    return FEWBIT_OK;
}

attn::Rows rows_of(const fewbit_heads *t) { return t == nullptr ? attn::Rows{} : attn::Rows{t->data, t->batch_stride, t->row_stride, t->head_stride}; }

fewbit_status fill(const fewbit_attention_shape *s, const Sizes &z, Params *p) {
    p->q_offsets = s->q_offsets;
    p->k_offsets = s->k_offsets;
    p->q_rows = z.q_rows;
    p->k_rows = z.k_rows;
    p->batch = s->batch;
    p->heads = s->heads;
    p->kv_heads = s->kv_heads;
    p->group = s->heads / s->kv_heads;
    p->dim = s->head_dim;
    p->q_len = static_cast<int>(s->q_len);
    p->k_len = static_cast<int>(s->k_len);
    p->causal = s->causal != 0;
    p->scale = s->scale;
    p->scale_log2 = s->scale * 1.4426950408889634f;
    static std::atomic<unsigned int *> cached[64];                    // per device
    int dev = 0;
    cudaError_t err = cudaGetDevice(&dev);
    // a thread that has not used the runtime yet (autograd's) has no context, which the tensor maps' encoder needs
    if (err == cudaSuccess) err = cudaSetDevice(dev);
    if (err != cudaSuccess) return cuda_status(err);
    unsigned int *at = dev < 64 ? cached[dev].load(std::memory_order_acquire) : nullptr;
    if (at == nullptr) {
        err = cudaGetSymbolAddress(reinterpret_cast<void **>(&at), g_attention_timeouts);
        if (err != cudaSuccess) return cuda_status(err);
        if (dev < 64) cached[dev].store(at, std::memory_order_release);
    }
    p->timeouts = at;
    p->sms = device_sm_count(&err);
    return cuda_status(err);
}

// The CTAs of a cluster that share one tile: 1, 2, 4 or 8, whichever should be done first, by the longest CTA or by the SMs'
// share of all work, counted in tiles of the long axis (`longest` of them for each of `tiles`; causal sequences have half
// the work, and the same longest CTA).  A CTA's start and end cost as much as ends.alone tiles, with a cluster's sums
// ends.joined.
struct Ends { int alone, joined; };
// dK, dV: 11000 and 20000 clocks against 2850 for a tile; the others have shorter ends and longer tiles by their chain of one
// tile after another.  Measured, in us.  Backward pass with dK's and dV's clusters of 1 / 2 / 4: 4 x 2048 rows of 16 heads on 4
// key heads, causal, 275 / 292 / 330; one of 16384 rows, 8 heads on 2, 1663 / 1608 / 1695.  Forward and backward pass with
// one CTA for a row tile against the clusters chosen here: one row on 8192 keys, 8 heads on 2, 92.7 and 85.7 against 25.7 and
// 35.4; 64 rows on 9000 keys, 4 heads, 102.9 and 99.0 against 27.3 and 41.2; 1024 rows, causal, 20.7 and 37.5 against 16.3 and
// 35.1; 4096 rows, causal, 59.9 and 120 against 47.7 and 119; 2 x 2048 rows stay with one: 35.0, with two 36.2.
constexpr Ends kDkvEnds = {4, 7};
constexpr Ends kDqEnds = {6, 9};
constexpr Ends kForwardEnds = {3, 7};

int choose_split(int64_t sms, int64_t tiles, int64_t longest, bool causal, int most, Ends ends) {
    int64_t best = INT64_MAX;
    int choice = 1;
    for (int split = 1; split <= most && (split == 1 || split <= longest); split *= 2) {
        const int64_t each = split == 1 ? ends.alone : ends.joined;
        const int64_t alone = (longest + split - 1) / split + each, shared = (tiles * longest / (causal ? 2 : 1) + tiles * split * each) / sms;
        const int64_t cost = alone > shared ? alone : shared;
        if (cost < best) {
            best = cost;
            choice = split;
        }
    }
    return choice;
}

fewbit_status run(attn::Kernel which, const fewbit_attention_shape *s, Params &p, int64_t tiles, int heads, void *stream) {
    p.tiles = static_cast<int>(p.q_offsets != nullptr && tiles == 0 ? 1 : tiles);   // packed rows of no sequence are there without any tile
    const unsigned grid = static_cast<unsigned>(static_cast<int64_t>(p.tiles) * heads * (s->batch + (p.q_offsets != nullptr)));   // one more for rows of no sequence
    if (grid == 0) return FEWBIT_OK;
    const cudaError_t err = (s->dtype == FEWBIT_F16 ? attn::launch_f16 : attn::launch_bf16)(which, s->head_dim > 64, p, grid, static_cast<cudaStream_t>(stream));
    if (err == cudaSuccess) g_launches.fetch_add(1, std::memory_order_relaxed);
    return cuda_status(err);
}

}  // namespace
}  // namespace fewbit

extern "C" {

fewbit_status fewbit_attention_fwd(const fewbit_attention_shape *s, const fewbit_heads *q, const fewbit_heads *k, const fewbit_heads *v,
                                   const fewbit_heads *out, float *lse, void *stream) {
    using namespace fewbit;
    Sizes z;
    if (const fewbit_status st = check_shape(s, &z); st != FEWBIT_OK) return st;
    if (z.batch == 0 || s->heads == 0 || z.q_rows == 0) return FEWBIT_OK;
    for (const fewbit_heads *t : {q, out})
        if (const fewbit_status st = check_tensor(t, z.q_rows, s->heads, z.batch); st != FEWBIT_OK) return st;
    for (const fewbit_heads *t : {k, v})
        if (const fewbit_status st = check_tensor(t, z.k_rows, s->kv_heads, z.batch); st != FEWBIT_OK) return st;
    if (lse == nullptr) return FEWBIT_ERR_INVALID_ARG;
    if (reinterpret_cast<uintptr_t>(lse) & 3) return FEWBIT_ERR_ALIGNMENT;
    Params p = {};
    fewbit_status st = fill(s, z, &p);
    if (st == FEWBIT_OK) st = encode(&p.q, q, s, z.q_rows, s->heads, z.batch);
    if (st == FEWBIT_OK && z.k_rows > 0) st = encode(&p.k, k, s, z.k_rows, s->kv_heads, z.batch);
    if (st == FEWBIT_OK && z.k_rows > 0) st = encode(&p.v, v, s, z.k_rows, s->kv_heads, z.batch);
    if (st != FEWBIT_OK) return st;
    p.out = rows_of(out);
    p.lse = lse;
    const int64_t row_tiles = (s->q_len + 2 * attn::kTile - 1) / (2 * attn::kTile), key_tiles = (s->k_len + attn::kTile - 1) / attn::kTile;
    p.split = choose_split(p.sms, row_tiles * s->heads * s->batch, key_tiles, p.causal, s->head_dim > 64 ? 8 : 4, kForwardEnds);
    return run(attn::Kernel::forward, s, p, row_tiles, s->heads, stream);
}

size_t fewbit_attention_workspace_bytes(const fewbit_attention_shape *s) {
    using namespace fewbit;
    Sizes z;
    if (check_shape(s, &z) != FEWBIT_OK) return 0;
    const size_t tiles = z.packed ? static_cast<size_t>(z.q_rows / attn::kTile + s->batch + 1) : static_cast<size_t>((s->q_len + attn::kTile - 1) / attn::kTile) * s->batch;
    return tiles * s->heads * attn::kStatBytes;
}

fewbit_status fewbit_attention_bwd(const fewbit_attention_shape *s, const fewbit_heads *grad_out, const fewbit_heads *q, const fewbit_heads *k,
                                   const fewbit_heads *v, const fewbit_heads *out, const float *lse, const fewbit_heads *grad_q,
                                   const fewbit_heads *grad_k, const fewbit_heads *grad_v, void *workspace, size_t workspace_bytes, void *stream) {
    using namespace fewbit;
    Sizes z;
    if (const fewbit_status st = check_shape(s, &z); st != FEWBIT_OK) return st;
    if (z.batch == 0 || s->heads == 0 || (z.q_rows == 0 && z.k_rows == 0)) return FEWBIT_OK;
    for (const fewbit_heads *t : {grad_out, q, out, grad_q})
        if (const fewbit_status st = check_tensor(t, z.q_rows, s->heads, z.batch); st != FEWBIT_OK) return st;
    for (const fewbit_heads *t : {k, v, grad_k, grad_v})
        if (const fewbit_status st = check_tensor(t, z.k_rows, s->kv_heads, z.batch); st != FEWBIT_OK) return st;
    const bool some = z.q_rows > 0;
    if (some && (lse == nullptr || workspace == nullptr)) return FEWBIT_ERR_INVALID_ARG;
    if ((reinterpret_cast<uintptr_t>(lse) & 3) || (reinterpret_cast<uintptr_t>(workspace) & 15)) return FEWBIT_ERR_ALIGNMENT;
    if (workspace_bytes < fewbit_attention_workspace_bytes(s)) return FEWBIT_ERR_ALLOC;
    Params p = {};
    fewbit_status st = fill(s, z, &p);
    if (st == FEWBIT_OK && some) st = encode(&p.q, q, s, z.q_rows, s->heads, z.batch);
    if (st == FEWBIT_OK && some) st = encode(&p.g, grad_out, s, z.q_rows, s->heads, z.batch);
    if (st == FEWBIT_OK && z.k_rows > 0) st = encode(&p.k, k, s, z.k_rows, s->kv_heads, z.batch);
    if (st == FEWBIT_OK && z.k_rows > 0) st = encode(&p.v, v, s, z.k_rows, s->kv_heads, z.batch);
    if (st != FEWBIT_OK) return st;
    p.o = rows_of(out);
    p.go = rows_of(grad_out);
    p.kin = rows_of(k);
    p.dq = rows_of(grad_q);
    p.dk = rows_of(grad_k);
    p.dv = rows_of(grad_v);
    p.lse = const_cast<float *>(lse);
    p.stat = static_cast<float *>(workspace);
    p.after_dq = some;
    const int64_t row_tiles = (s->q_len + attn::kTile - 1) / attn::kTile, key_tiles = (s->k_len + attn::kTile - 1) / attn::kTile;
    p.split = choose_split(p.sms, row_tiles * s->heads * s->batch, key_tiles, p.causal, s->head_dim > 64 ? 8 : 4, kDqEnds);
    if (some) st = run(attn::Kernel::dq, s, p, row_tiles, s->heads, stream);
    if (st != FEWBIT_OK || z.k_rows == 0) return st;
    p.split = choose_split(p.sms, key_tiles * s->kv_heads * s->batch, row_tiles * p.group, p.causal, 4, kDkvEnds);
    return run(attn::Kernel::dkv, s, p, key_tiles, s->kv_heads, stream);
}

fewbit_status fewbit_attention_timeout_count(uint64_t *count) {
    using namespace fewbit;
    if (count == nullptr) return FEWBIT_ERR_INVALID_ARG;
    unsigned int n = 0;
    cudaError_t err = cudaDeviceSynchronize();                        // (a copy alone does not wait for non-blocking streams)
    if (err == cudaSuccess) err = cudaMemcpyFromSymbol(&n, g_attention_timeouts, sizeof(n));
    *count = n;
    return cuda_status(err);
}

}  // extern "C"
