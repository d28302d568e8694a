// Argument marshalling of the training operators for PyTorch: checks, output and workspace allocation, the call of the C ABI.
// The same as operators.py would do through ctypes, in a few microseconds: a small tensor's kernel takes no longer.
#include <torch/extension.h>

#include <ATen/MemoryOverlap.h>
#include <c10/cuda/CUDAGuard.h>
#include <c10/cuda/CUDAStream.h>

#include <limits>
#include <optional>
#include <variant>
#include <vector>

#include "fewbit.h"

namespace {

using at::Tensor;
using Optional = std::optional<Tensor>;

// FewbitError(status, where)
struct StatusError {
    fewbit_status status;
    const char *where;
};
void check(fewbit_status s, const char *where) {
    if (s != FEWBIT_OK) throw StatusError{s, where};
}
[[noreturn]] void refuse(const char *what) { throw py::value_error(what); }

fewbit_dtype dtype_of(const Tensor &t) {
    switch (t.scalar_type()) {
    case at::kFloat: return FEWBIT_F32;
    case at::kBFloat16: return FEWBIT_BF16;
    case at::kHalf: return FEWBIT_F16;
    default: refuse("tensors must be float32, bfloat16 or float16");
    }
}
void *stream_of(const Tensor &t) { return c10::cuda::getCurrentCUDAStream(t.get_device()).stream(); }

// A size that the C structs hold in 31 bits; more than that (a view expanded to it) would come out as another size.
int size_of(int64_t n) {
    if (n > INT32_MAX) refuse("the tensors are too large: batch, heads and head_dim are counted in 31 bits");
    return static_cast<int>(n);
}
// (batch, length, heads, head_dim) or (rows, heads, head_dim)
fewbit_heads heads_of(const Tensor &t) {
    const auto st = t.strides();
    const int64_t n = t.dim();
    if (t.size(n - 1) > 1 && st[n - 1] != 1) refuse("the elements of one head must be contiguous");
    return n == 4 ? fewbit_heads{t.data_ptr(), st[0], st[1], st[2]} : fewbit_heads{t.data_ptr(), 0, st[0], st[1]};
}
void like(const Tensor &t, const Tensor &model, const char *what) {
    if (t.sizes() != model.sizes() || t.scalar_type() != model.scalar_type() || t.device() != model.device()) refuse(what);
}
void dense(const Tensor &t, const char *what) {
    if (!t.is_cuda() || !t.is_contiguous()) refuse(what);
}
const float *vector_of(const Optional &w, const Tensor &q, int64_t n) {
    if (!w) return nullptr;
    if (w->scalar_type() != at::kFloat || w->device() != q.device() || w->dim() != 1 || w->numel() != n || !w->is_contiguous())
        refuse("q_weight and k_weight must be contiguous float32 vectors of head_dim values on the device of q");
    return w->data_ptr<float>();
}

fewbit_qk_shape qk_shape(const Tensor &q, const Tensor &k, const Optional &qw, const Optional &kw, const Optional &cos, const Optional &sin,
                         const Optional &positions, double eps, bool interleaved) {
    if (q.dim() != 4 || k.dim() != 4 || !q.is_cuda()) refuse("q and k must be (batch, length, heads, head_dim) CUDA tensors");
    if (k.size(0) != q.size(0) || k.size(1) != q.size(1) || k.size(3) != q.size(3) || k.scalar_type() != q.scalar_type() || k.device() != q.device())
        refuse("q and k must have one type and device, and the same batch, length and head_dim");
    fewbit_qk_shape s = {};
    s.dtype = dtype_of(q);
    s.batch = size_of(q.size(0));
    s.length = q.size(1);
    s.heads = size_of(q.size(2));
    s.kv_heads = size_of(k.size(2));
    s.head_dim = size_of(q.size(3));
    s.interleaved = interleaved;
    s.eps = static_cast<float>(eps);
    s.q_weight = vector_of(qw, q, q.size(3));
    s.k_weight = vector_of(kw, q, q.size(3));
    if (cos.has_value() != sin.has_value()) refuse("cos and sin come together");
    if (cos) {
        for (const Tensor *t : {&*cos, &*sin})
            if (t->dim() != 2 || t->sizes() != cos->sizes() || !t->is_contiguous() || t->scalar_type() != at::kFloat || t->device() != q.device())
                refuse("cos and sin must be contiguous float32 (rows, rotary_dim / 2) tables on the device of q");
        s.table_rows = cos->size(0);
        s.rotary_dim = static_cast<int>(2 * std::min<int64_t>(cos->size(1), INT32_MAX / 2));
        s.cos = cos->data_ptr<float>();
        s.sin = sin->data_ptr<float>();
    }
    if (positions) {
        const auto t = positions->scalar_type();
        if (positions->dim() != 2 || positions->size(0) != q.size(0) || positions->size(1) != q.size(1) || (t != at::kLong && t != at::kInt) ||
            !positions->is_contiguous() || positions->device() != q.device())
            refuse("positions must be a contiguous (batch, length) tensor of int32 or int64 on the device of q");
        s.positions = positions->data_ptr();
        s.positions_are_64bit = t == at::kLong;
    }
    return s;
}

Tensor output(const Optional &given, const Tensor &model) {
    if (!given) return at::empty(model.sizes(), model.options());
    like(*given, model, "out does not match q and k");
    return *given;
}
// Tensors that a call writes, `a` for the queries and `b` for the keys, against all that it reads: an output may be its own side's input,
// element for element, and share no other memory (as far as ATen tells: not for views with gaps).
void no_overlap(const Tensor &a, const Tensor &b, std::initializer_list<std::reference_wrapper<const Tensor>> of_a, std::initializer_list<std::reference_wrapper<const Tensor>> of_b) {
    const char *what = "an output overlaps itself, the other output or an input in part";
    for (const Tensor *t : {&a, &b})
        if (at::has_internal_overlap(*t) == at::MemOverlap::Yes) refuse(what);
    auto shares = [&](const Tensor &x, const Tensor &y, bool own_side) {
        const auto s = at::get_overlap_status(x, y);
        return s == at::MemOverlapStatus::Partial || (s == at::MemOverlapStatus::Full && !own_side);
    };
    if (shares(a, b, false)) refuse(what);
    for (const Tensor &t : of_a)
        if (shares(a, t, true) || shares(b, t, false)) refuse(what);
    for (const Tensor &t : of_b)
        if (shares(b, t, true) || shares(a, t, false)) refuse(what);
}

std::tuple<Tensor, Tensor> qk_norm_rope_fwd(const Tensor &q, const Tensor &k, const Optional &qw, const Optional &kw, const Optional &cos, const Optional &sin,
                                            const Optional &positions, double eps, bool interleaved, const Optional &q_out, const Optional &k_out) {
    const fewbit_qk_shape s = qk_shape(q, k, qw, kw, cos, sin, positions, eps, interleaved);
    const c10::cuda::OptionalCUDAGuard guard(q.device());
    Tensor a = output(q_out, q), b = output(k_out, k);
    if (q_out || k_out) no_overlap(a, b, {q}, {k});
    const fewbit_heads h[4] = {heads_of(q), heads_of(k), heads_of(a), heads_of(b)};
    check(fewbit_qk_norm_rope_fwd(&s, &h[0], &h[1], &h[2], &h[3], stream_of(q)), "fewbit_qk_norm_rope_fwd");
    return {a, b};
}

std::tuple<Tensor, Tensor, Optional, Optional> qk_norm_rope_bwd(const Tensor &gq, const Tensor &gk, const Tensor &q, const Tensor &k, const Optional &qw,
                                                                const Optional &kw, const Optional &cos, const Optional &sin, const Optional &positions,
                                                                double eps, bool interleaved, bool weight_grads, const Optional &q_out, const Optional &k_out) {
    const fewbit_qk_shape s = qk_shape(q, k, qw, kw, cos, sin, positions, eps, interleaved);
    like(gq, q, "the gradients do not match q and k");
    like(gk, k, "the gradients do not match q and k");
    const c10::cuda::OptionalCUDAGuard guard(q.device());
    Tensor a = output(q_out, q), b = output(k_out, k), ws;
    if (q_out || k_out) no_overlap(a, b, {q, gq}, {k, gk});
    Optional dqw, dkw;
    size_t bytes = 0;
    if (weight_grads) {
        const auto f32 = q.options().dtype(at::kFloat);
        dqw = at::empty({q.size(3)}, f32);
        dkw = at::empty({q.size(3)}, f32);
        bytes = fewbit_qk_norm_rope_workspace_bytes(&s);
        ws = at::empty({static_cast<int64_t>(bytes)}, q.options().dtype(at::kByte));
    }
    const fewbit_heads h[6] = {heads_of(gq), heads_of(gk), heads_of(q), heads_of(k), heads_of(a), heads_of(b)};
    check(fewbit_qk_norm_rope_bwd(&s, &h[0], &h[1], &h[2], &h[3], &h[4], &h[5], dqw ? dqw->data_ptr<float>() : nullptr, dkw ? dkw->data_ptr<float>() : nullptr,
                                  bytes ? ws.data_ptr() : nullptr, bytes, stream_of(q)),
          "fewbit_qk_norm_rope_bwd");
    return {a, b, dqw, dkw};
}

struct Attention {
    fewbit_attention_shape s = {};
    std::vector<int64_t> stats;                                       // shape of lse
};
Attention attention_shape(const Tensor &q, const Tensor &k, const Tensor &v, bool causal, std::optional<double> scale, const Optional &q_offsets,
                          const Optional &k_offsets, std::optional<int64_t> max_q, std::optional<int64_t> max_k) {
    if ((q.scalar_type() != at::kBFloat16 && q.scalar_type() != at::kHalf) || !q.is_cuda()) refuse("attention takes bfloat16 or float16 CUDA tensors");
    like(v, k, "k and v must have one shape, type and device");
    if (k.scalar_type() != q.scalar_type() || k.device() != q.device()) refuse("q, k and v must have one type and device");
    const bool packed = q_offsets.has_value();
    if (packed != k_offsets.has_value() || packed != max_q.has_value() || packed != max_k.has_value())
        refuse("packed sequences need q_offsets, k_offsets, max_q_len and max_k_len, others none of them");
    const int64_t n = packed ? 3 : 4;
    if (q.dim() != n || k.dim() != n) refuse(packed ? "packed sequences are (rows, heads, head_dim) tensors" : "q, k and v must be (batch, length, heads, head_dim) tensors");
    if (k.size(n - 1) != q.size(n - 1) || (!packed && k.size(0) != q.size(0))) refuse("q, k and v must have the same batch and head_dim");
    Attention a;
    fewbit_attention_shape &s = a.s;
    s.dtype = dtype_of(q);
    s.heads = size_of(q.size(n - 2));
    s.kv_heads = size_of(k.size(n - 2));
    s.head_dim = size_of(q.size(n - 1));
    s.causal = causal;
    s.scale = static_cast<float>(scale ? *scale : 1.0 / std::sqrt(static_cast<double>(q.size(n - 1))));
    if (!packed) {
        s.batch = size_of(q.size(0));
        s.q_len = q.size(1);
        s.k_len = k.size(1);
        a.stats = {q.size(0), q.size(2), q.size(1)};
        return a;
    }
    for (const Tensor *o : {&*q_offsets, &*k_offsets})
        if (o->scalar_type() != at::kInt || o->device() != q.device() || o->dim() != 1 || o->numel() < 1 || o->numel() != q_offsets->numel() || !o->is_contiguous())
            refuse("q_offsets and k_offsets must be contiguous vectors of batch + 1 int32 values on the device of q");
    s.batch = size_of(q_offsets->numel() - 1);
    s.q_rows = q.size(0);
    s.k_rows = k.size(0);
    s.q_len = std::min(*max_q, s.q_rows);
    s.k_len = std::min(*max_k, s.k_rows);
    s.q_offsets = q_offsets->data_ptr<int32_t>();
    s.k_offsets = k_offsets->data_ptr<int32_t>();
    a.stats = {q.size(1), q.size(0)};
    return a;
}

fewbit_attention_scores scores_of(const Attention &a, const Tensor &q, const Tensor &k, std::optional<double> cap, const Optional &slopes, const Optional &distance_bias,
                                  const Optional &prefix_lens, const Optional &q_documents, const Optional &k_documents) {
    fewbit_attention_scores c = {};
    auto is = [&](const Tensor &t, at::ScalarType type) { return t.scalar_type() == type && t.device() == q.device() && t.is_contiguous(); };
    if (cap) {
        if (!(*cap >= 0)) refuse("cap must not be negative");
        c.cap = static_cast<float>(*cap);
        if (*cap > 0 && c.cap == 0) c.cap = std::numeric_limits<float>::min();   // (0 is no cap: the library refuses this one, as every cap below its range)
    }
    if (slopes) {
        if (!is(*slopes, at::kFloat) || slopes->dim() != 1 || slopes->size(0) != a.s.heads) refuse("slopes must be a contiguous float32 vector with a value for each head of q, on its device");
        c.slopes = slopes->data_ptr<float>();
    }
    if (distance_bias) {
        const Tensor &t = *distance_bias;
        if (!is(t, at::kFloat) || t.dim() != 2 || t.size(0) != a.s.heads || t.size(1) % 2 != 1 || t.size(1) < 3 || t.size(1) > 2 * FEWBIT_MAX_DISTANCE + 1)
            refuse("distance_bias must be a contiguous float32 (heads, 2 R + 1) tensor on the device of q, R from 1 to 4096");
        c.distance_bias = t.data_ptr<float>();
        c.max_distance = static_cast<int>(t.size(1) / 2);
    }
    if (prefix_lens) {
        if (!a.s.causal) refuse("prefix_lens are for causal attention");
        if (!is(*prefix_lens, at::kInt) || prefix_lens->dim() != 1 || prefix_lens->size(0) != a.s.batch) refuse("prefix_lens must be a contiguous int32 vector with a value for each sequence, on the device of q");
        c.prefix_lens = prefix_lens->data_ptr<int32_t>();
    }
    if (q_documents.has_value() != k_documents.has_value()) refuse("q_documents and k_documents come together");
    if (q_documents) {
        const int64_t lead = q.dim() - 2;                             // (batch, length) or (rows)
        if (!is(*q_documents, at::kInt) || !is(*k_documents, at::kInt) || q_documents->sizes() != q.sizes().slice(0, lead) || k_documents->sizes() != k.sizes().slice(0, lead))
            refuse("q_documents and k_documents must be contiguous int32 tensors with a value for each row of q and of k, on their device");
        if (q_documents->numel() > 0 && k_documents->numel() > 0) {   // (an empty tensor's pointer is NULL; without rows or keys there is nothing to tell apart)
            c.q_documents = q_documents->data_ptr<int32_t>();
            c.k_documents = k_documents->data_ptr<int32_t>();
        }
    }
    return c;
}

std::tuple<Tensor, Tensor> attention_fwd(const Tensor &q, const Tensor &k, const Tensor &v, bool causal, std::optional<double> scale, const Optional &q_offsets,
                                         const Optional &k_offsets, std::optional<int64_t> max_q, std::optional<int64_t> max_k, std::optional<double> cap,
                                         const Optional &slopes, const Optional &distance_bias, const Optional &prefix_lens, const Optional &q_documents,
                                         const Optional &k_documents) {
    const Attention a = attention_shape(q, k, v, causal, scale, q_offsets, k_offsets, max_q, max_k);
    const fewbit_attention_scores c = scores_of(a, q, k, cap, slopes, distance_bias, prefix_lens, q_documents, k_documents);
    const c10::cuda::OptionalCUDAGuard guard(q.device());
    Tensor out = at::empty(q.sizes(), q.options()), lse = at::empty(a.stats, q.options().dtype(at::kFloat));
    const fewbit_heads h[4] = {heads_of(q), heads_of(k), heads_of(v), heads_of(out)};
    check(fewbit_attention_scores_fwd(&a.s, &c, &h[0], &h[1], &h[2], &h[3], lse.data_ptr<float>(), stream_of(q)), "fewbit_attention_fwd");
    return {out, lse};
}

std::vector<Tensor> attention_bwd(const Tensor &g, const Tensor &q, const Tensor &k, const Tensor &v, const Tensor &out, const Tensor &lse,
                                  bool causal, std::optional<double> scale, const Optional &q_offsets, const Optional &k_offsets,
                                  std::optional<int64_t> max_q, std::optional<int64_t> max_k, std::optional<double> cap, const Optional &slopes,
                                  const Optional &distance_bias, const Optional &prefix_lens, const Optional &q_documents, const Optional &k_documents,
                                  bool bias_grad) {
    const Attention a = attention_shape(q, k, v, causal, scale, q_offsets, k_offsets, max_q, max_k);
    const fewbit_attention_scores c = scores_of(a, q, k, cap, slopes, distance_bias, prefix_lens, q_documents, k_documents);
    like(g, q, "grad_out must have the shape and type of the output");
    like(out, q, "out must be what the forward pass gave");
    if (lse.sizes() != at::IntArrayRef(a.stats) || lse.scalar_type() != at::kFloat || lse.device() != q.device() || !lse.is_contiguous())
        refuse("lse must be what the forward pass gave");
    const c10::cuda::OptionalCUDAGuard guard(q.device());
    // without query heads the library has nothing to do, and the sums over them are zero
    const bool none = a.s.heads == 0;
    Tensor dq = at::empty(q.sizes(), q.options());
    Tensor dk = none ? at::zeros(k.sizes(), k.options()) : at::empty(k.sizes(), k.options());
    Tensor dv = none ? at::zeros(v.sizes(), v.options()) : at::empty(v.sizes(), v.options());
    bias_grad = bias_grad && distance_bias;
    Tensor db;
    if (bias_grad) db = none ? at::zeros(distance_bias->sizes(), distance_bias->options()) : at::empty(distance_bias->sizes(), distance_bias->options());
    const size_t bytes = fewbit_attention_scores_workspace_bytes(&a.s, &c, bias_grad);
    Tensor ws = at::empty({static_cast<int64_t>(bytes)}, q.options().dtype(at::kByte));
    const fewbit_heads h[8] = {heads_of(g), heads_of(q), heads_of(k), heads_of(v), heads_of(out), heads_of(dq), heads_of(dk), heads_of(dv)};
    check(fewbit_attention_scores_bwd(&a.s, &c, &h[0], &h[1], &h[2], &h[3], &h[4], lse.data_ptr<float>(), &h[5], &h[6], &h[7],
                                      bias_grad && !none ? db.data_ptr<float>() : nullptr, ws.data_ptr(), bytes, stream_of(q)),
          "fewbit_attention_bwd");
    if (bias_grad) return {dq, dk, dv, db};
    return {dq, dk, dv};
}

Tensor relative_bias_fwd(const Tensor &table, int64_t max_distance, bool bidirectional) {
    dense(table, "table must be a contiguous CUDA tensor");
    if (table.dim() != 2) refuse("table must be (buckets, heads)");
    const fewbit_dtype dtype = dtype_of(table);
    const int buckets = size_of(table.size(0)), heads = size_of(table.size(1));
    if (max_distance < 1 || max_distance > FEWBIT_MAX_DISTANCE) refuse("max_distance must be from 1 to 4096");
    const c10::cuda::OptionalCUDAGuard guard(table.device());
    Tensor bias = at::empty({heads, 2 * max_distance + 1}, table.options().dtype(at::kFloat));
    check(fewbit_relative_bias_fwd(table.data_ptr(), buckets, heads, static_cast<int>(max_distance), bidirectional, dtype, bias.data_ptr<float>(), stream_of(table)),
          "fewbit_relative_bias_fwd");
    return bias;
}
Tensor relative_bias_bwd(const Tensor &grad, const Tensor &table, bool bidirectional) {
    dense(grad, "grad_distance_bias must be a contiguous CUDA tensor");
    if (table.dim() != 2 || grad.dim() != 2 || grad.scalar_type() != at::kFloat || grad.device() != table.device() || grad.size(0) != table.size(1) || grad.size(1) % 2 != 1 ||
        grad.size(1) < 3 || grad.size(1) > 2 * FEWBIT_MAX_DISTANCE + 1)
        refuse("grad_distance_bias must be float32 (heads, 2 R + 1) for a table (buckets, heads) on the same device");
    const fewbit_dtype dtype = dtype_of(table);
    const int buckets = size_of(table.size(0)), heads = size_of(table.size(1));
    const c10::cuda::OptionalCUDAGuard guard(grad.device());
    Tensor out = at::empty(table.sizes(), grad.options().dtype(table.scalar_type()));
    check(fewbit_relative_bias_bwd(grad.data_ptr<float>(), buckets, heads, static_cast<int>(grad.size(1) / 2), bidirectional, dtype, out.data_ptr(), stream_of(grad)),
          "fewbit_relative_bias_bwd");
    return out;
}

// Dropout's numbers: `seed` is an integer or one int64 value on the device of the tensors.
using Seed = std::variant<uint64_t, Tensor>;
fewbit_dropout_options drop_of(double p, const Seed &seed, int64_t place, const Tensor &x) {
    if (!(p >= 0.0 && p < 1.0)) refuse("p must be at least 0 and below 1");
    if (place < 0 || place > UINT32_MAX) refuse("place must be a whole number of 32 bits");
    fewbit_dropout_options o = {p, 0, nullptr, static_cast<uint32_t>(place)};
    if (const Tensor *t = std::get_if<Tensor>(&seed)) {
        if (t->scalar_type() != at::kLong || t->numel() != 1 || t->device() != x.device()) refuse("seed must be an integer or one int64 value on the device of the tensors");
        o.seed_device = t->data_ptr<int64_t>();
    } else {
        o.seed = std::get<uint64_t>(seed);
    }
    return o;
}
// An output against the inputs of its call: one of them element for element, or no shared memory at all.
void whole_or_none(const Tensor &out, std::initializer_list<const Tensor *> inputs) {
    for (const Tensor *t : inputs)
        if (t != nullptr && at::get_overlap_status(out, *t) == at::MemOverlapStatus::Partial) refuse("out overlaps an input in part");
}

Tensor dropout_fwd(const Tensor &x, double p, const Seed &seed, int64_t place, const Optional &residual, const Optional &out) {
    dense(x, "x must be a contiguous CUDA tensor");
    const fewbit_dtype dtype = dtype_of(x);
    const fewbit_dropout_options o = drop_of(p, seed, place, x);
    if (residual) {
        like(*residual, x, "residual must have the shape, type and device of x");
        dense(*residual, "residual must be contiguous");
    }
    const c10::cuda::OptionalCUDAGuard guard(x.device());
    Tensor y = out ? *out : at::empty(x.sizes(), x.options());
    if (out) {
        like(y, x, "out must have the shape, type and device of x");
        dense(y, "out must be contiguous");
        whole_or_none(y, {&x, residual ? &*residual : nullptr});
    }
    check(fewbit_dropout_fwd(x.data_ptr(), residual ? residual->data_ptr() : nullptr, y.data_ptr(), x.numel(), dtype, &o, stream_of(x)), "fewbit_dropout_fwd");
    return y;
}
Tensor dropout_bwd(const Tensor &g, double p, const Seed &seed, int64_t place, const Optional &out) {
    dense(g, "grad_out must be a contiguous CUDA tensor");
    const fewbit_dtype dtype = dtype_of(g);
    const fewbit_dropout_options o = drop_of(p, seed, place, g);
    const c10::cuda::OptionalCUDAGuard guard(g.device());
    Tensor y = out ? *out : at::empty(g.sizes(), g.options());
    if (out) {
        like(y, g, "out must have the shape, type and device of grad_out");
        dense(y, "out must be contiguous");
        whole_or_none(y, {&g});
    }
    check(fewbit_dropout_bwd(g.data_ptr(), y.data_ptr(), g.numel(), dtype, &o, stream_of(g)), "fewbit_dropout_bwd");
    return y;
}

fewbit_norm_shape norm_shape(const Tensor &x, const Optional &weight, double eps, double p, const Seed &seed, int64_t place) {
    dense(x, "the tensors must be contiguous and on a CUDA device");
    if (x.dim() < 1) refuse("the tensors must have a last dimension");
    fewbit_norm_shape s = {};
    s.dtype = dtype_of(x);
    s.width = x.size(x.dim() - 1);
    s.rows = 1;
    for (int64_t i = 0; i + 1 < x.dim(); ++i) s.rows *= x.size(i);
    s.eps = static_cast<float>(eps);
    s.dropout = drop_of(p, seed, place, x);
    if (weight) {
        if (weight->scalar_type() != at::kFloat || weight->device() != x.device() || weight->dim() != 1 || weight->numel() != s.width || !weight->is_contiguous())
            refuse("weight must be a contiguous float32 vector with a value for each element of the last dimension, on the device of the tensors");
        s.weight = weight->data_ptr<float>();
    }
    return s;
}
std::vector<Tensor> add_rms_norm_fwd(const Tensor &x, const Optional &residual, const Optional &weight, double eps, double p, const Seed &seed, int64_t place,
                                     std::optional<int64_t> bits) {
    const fewbit_norm_shape s = norm_shape(x, weight, eps, p, seed, place);
    if (bits && *bits != 8) refuse("bits must be 8 or None");
    if (residual) {
        like(*residual, x, "residual must have the shape, type and device of x");
        dense(*residual, "residual must be contiguous");
    }
    const c10::cuda::OptionalCUDAGuard guard(x.device());
    const bool sum = residual || p > 0.0;                             // else h is x
    Tensor h = sum ? at::empty(x.sizes(), x.options()) : x;
    Tensor y = at::empty(x.sizes(), bits ? x.options().dtype(at::kFloat8_e4m3fn) : x.options()), scale;
    if (bits) scale = at::empty(x.sizes().slice(0, x.dim() - 1), x.options().dtype(at::kFloat));
    check(fewbit_add_rms_norm_fwd(&s, x.data_ptr(), residual ? residual->data_ptr() : nullptr, sum ? h.data_ptr() : nullptr, y.data_ptr(),
                                  bits ? scale.data_ptr<float>() : nullptr, bits ? 8 : 0, stream_of(x)),
          "fewbit_add_rms_norm_fwd");
    if (bits) return {y, scale, h};
    return {y, h};
}
std::tuple<Optional, Optional, Optional> add_rms_norm_bwd(const Tensor &grad_y, const Optional &grad_h, const Tensor &h, const Optional &weight, double eps, double p,
                                                          const Seed &seed, int64_t place, bool x_grad, bool residual_grad, bool weight_grad) {
    const fewbit_norm_shape s = norm_shape(h, weight, eps, p, seed, place);
    like(grad_y, h, "grad_y must have the shape, type and device of h");
    dense(grad_y, "grad_y must be contiguous");
    if (grad_h) {
        like(*grad_h, h, "grad_h must have the shape, type and device of h");
        dense(*grad_h, "grad_h must be contiguous");
    }
    const c10::cuda::OptionalCUDAGuard guard(h.device());
    // without dropout the two gradients are one
    const bool dropped = p > 0.0;
    Optional gx, gr, gw;
    if (residual_grad || (x_grad && !dropped)) gr = at::empty(h.sizes(), h.options());
    if (x_grad && dropped) gx = at::empty(h.sizes(), h.options());
    Tensor ws;
    size_t bytes = 0;
    if (weight_grad) {
        gw = at::empty({s.width}, h.options().dtype(at::kFloat));
        bytes = fewbit_add_rms_norm_workspace_bytes(&s);
        ws = at::empty({static_cast<int64_t>(bytes)}, h.options().dtype(at::kByte));
    }
    check(fewbit_add_rms_norm_bwd(&s, grad_y.data_ptr(), grad_h ? grad_h->data_ptr() : nullptr, h.data_ptr(), gx ? gx->data_ptr() : nullptr,
                                  gr ? gr->data_ptr() : nullptr, gw ? gw->data_ptr<float>() : nullptr, bytes ? ws.data_ptr() : nullptr, bytes, stream_of(h)),
          "fewbit_add_rms_norm_bwd");
    if (x_grad && !dropped) gx = gr;
    if (!residual_grad) gr.reset();
    return {gx, gr, gw};
}

// What a program keeps for its steps: the tensors, not where they lie (`p.data = ...` puts other memory under a parameter).
class AdamW {
public:
    AdamW(std::vector<Tensor> params_, std::vector<Tensor> m_, std::vector<Tensor> v_, std::optional<std::vector<Tensor>> ms_, std::optional<std::vector<Tensor>> vs_,
          std::optional<std::vector<Tensor>> masters_)
        : params(std::move(params_)), m(std::move(m_)), v(std::move(v_)), ms(std::move(ms_)), vs(std::move(vs_)), masters(std::move(masters_)) {
        const size_t n = params.size();
        if (n == 0 || m.size() != n || v.size() != n || (ms && ms->size() != n) || (vs && vs->size() != n) || (masters && masters->size() != n))
            refuse("every list must have one tensor for each parameter, and there must be one");
        if (ms.has_value() != vs.has_value()) refuse("the scales of both moments come together");
        bits = ms ? 8 : 32;
        dtype = dtype_of(params[0]);
        type = params[0].scalar_type();
        device = params[0].device();
        if (masters && dtype == FEWBIT_F32) refuse("float32 parameters need no master copy");
        descriptions();
    }
    void step(const std::vector<Tensor> &grads, int64_t step, double lr, double beta1, double beta2, double eps, double weight_decay, int64_t seed,
              const Optional &grad_scale) const {
        if (grads.size() != params.size()) refuse("one gradient for each parameter is needed");
        const std::vector<fewbit_adamw_tensor> descs = descriptions();
        std::vector<const void *> pointers(grads.size());
        for (size_t i = 0; i < grads.size(); ++i) {
            const Tensor &g = grads[i];
            if (g.scalar_type() != type || g.device() != device || static_cast<uint64_t>(g.numel()) != descs[i].n || !g.is_contiguous())
                refuse("gradients must be contiguous tensors of the parameters' type, device and sizes");
            pointers[i] = g.data_ptr();
        }
        if (grad_scale && (grad_scale->scalar_type() != at::kFloat || grad_scale->device() != device || grad_scale->numel() != 1))
            refuse("grad_scale must be one float32 value on the device of the parameters");
        const fewbit_adamw_options o = {lr, beta1, beta2, eps, weight_decay, step, grad_scale ? grad_scale->data_ptr<float>() : nullptr,
                                        static_cast<uint32_t>(seed), bits, dtype};
        const c10::cuda::OptionalCUDAGuard guard(device);
        check(fewbit_adamw_step(descs.data(), pointers.data(), static_cast<int>(descs.size()), &o, c10::cuda::getCurrentCUDAStream(device.index()).stream()),
              "fewbit_adamw_step");
    }
    size_t size() const { return params.size(); }
    std::vector<Tensor> tensors() const {
        std::vector<Tensor> all;
        for (auto *x : {&params, &m, &v}) all.insert(all.end(), x->begin(), x->end());
        for (auto *x : {&ms, &vs, &masters})
            if (*x) all.insert(all.end(), (*x)->begin(), (*x)->end());
        return all;
    }
    int bits;
    at::Device device = at::kCPU;

private:
    std::vector<fewbit_adamw_tensor> descriptions() const {
        auto pointer = [&](const Tensor &t, at::ScalarType want, int64_t numel) {
            if (t.device() != device || !t.is_cuda() || t.scalar_type() != want || t.numel() != numel || !t.is_contiguous())
                refuse("parameters, moments (float32, or float8_e4m3fn with a float32 scale for each 256 elements) and masters (float32) must be contiguous CUDA "
                       "tensors of one device and matching sizes");
            return t.data_ptr();
        };
        const auto state = bits == 8 ? at::kFloat8_e4m3fn : at::kFloat;
        std::vector<fewbit_adamw_tensor> descs(params.size());
        for (size_t i = 0; i < descs.size(); ++i) {
            const int64_t numel = params[i].numel(), blocks = (numel + FEWBIT_ADAMW_BLOCK - 1) / FEWBIT_ADAMW_BLOCK;
            descs[i] = {pointer(params[i], type, numel), pointer(m[i], state, numel), pointer(v[i], state, numel),
                        ms ? static_cast<float *>(pointer((*ms)[i], at::kFloat, blocks)) : nullptr,
                        vs ? static_cast<float *>(pointer((*vs)[i], at::kFloat, blocks)) : nullptr,
                        masters ? static_cast<float *>(pointer((*masters)[i], at::kFloat, numel)) : nullptr, static_cast<uint64_t>(numel)};
        }
        return descs;
    }
    fewbit_dtype dtype;
    at::ScalarType type;
    std::vector<Tensor> params, m, v;
    std::optional<std::vector<Tensor>> ms, vs, masters;
};

}  // namespace

PYBIND11_MODULE(TORCH_EXTENSION_NAME, m) {
    py::register_exception_translator([](std::exception_ptr p) {
        try {
            if (p) std::rethrow_exception(p);
        } catch (const StatusError &e) {
            const py::object type = py::module_::import("paper_2202_00441_b200.binding").attr("FewbitError");
            const py::object error = type(static_cast<int>(e.status), e.where);
            PyErr_SetObject(type.ptr(), error.ptr());
        }
    });
    m.def("qk_norm_rope_fwd", &qk_norm_rope_fwd);
    m.def("qk_norm_rope_bwd", &qk_norm_rope_bwd);
    m.def("attention_fwd", &attention_fwd);
    m.def("attention_bwd", &attention_bwd);
    m.def("relative_bias_fwd", &relative_bias_fwd);
    m.def("relative_bias_bwd", &relative_bias_bwd);
    m.def("dropout_fwd", &dropout_fwd);
    m.def("dropout_bwd", &dropout_bwd);
    m.def("add_rms_norm_fwd", &add_rms_norm_fwd);
    m.def("add_rms_norm_bwd", &add_rms_norm_bwd);
    py::class_<AdamW>(m, "AdamWTensors", "The parameters and moments of fewbit_adamw_step, made once and updated in place by every step; keeps them alive.")
        .def(py::init<std::vector<Tensor>, std::vector<Tensor>, std::vector<Tensor>, std::optional<std::vector<Tensor>>, std::optional<std::vector<Tensor>>,
                      std::optional<std::vector<Tensor>>>())
        .def("step", &AdamW::step)
        .def("tensors", &AdamW::tensors)
        .def("__len__", &AdamW::size)
        .def_readonly("bits", &AdamW::bits)
        .def_property_readonly("device", [](const AdamW &a) { return a.device; });
}
