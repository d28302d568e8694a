"""Drop-in activation modules over the C ABI (Listing 1 as a PyTorch layer), and attention and the head norm with
rotation as differentiable functions.

``FewBitActivation("gelu", bits=3)`` replaces ``nn.GELU()``: the forward pass
returns the exact activation, autograd keeps only ``bits`` bits per element
(the packed interval codes) instead of the input, and the backward pass
multiplies the incoming gradient by the level of each element's interval.
Only argument marshalling happens here; both passes run in the CUDA library.
"""
from __future__ import annotations

import torch
from torch import nn
from torch.autograd.function import once_differentiable

from .binding import Table, fewbit_bwd, fewbit_fwd, fewbit_fwd_bias, fewbit_table_create, fewbit_table_create_folded
from .operators import (
    fewbit_relative_bias_bwd, fewbit_relative_bias_fwd,
    fewbit_add_rms_norm_bwd, fewbit_add_rms_norm_fwd, fewbit_attention_bwd, fewbit_attention_fwd, fewbit_dropout_bwd, fewbit_dropout_fwd,
    fewbit_qk_norm_rope_bwd, fewbit_qk_norm_rope_fwd,
)


def _flat_aligned(t: torch.Tensor) -> torch.Tensor:
    t = t.contiguous().view(-1)
    if t.data_ptr() % 32:                 # a view into the middle of a buffer: the library wants 32-byte alignment
        t = t.clone()
    return t


class _FewBitFunction(torch.autograd.Function):
    @staticmethod
    def forward(ctx, x: torch.Tensor, table: Table):
        if x.dtype not in (torch.float32, torch.bfloat16, torch.float16) or not x.is_cuda:
            raise TypeError("FewBitActivation needs a CUDA tensor of dtype float32, bfloat16 or float16")
        y, packed = fewbit_fwd(table, _flat_aligned(x))
        ctx.table = table
        ctx.save_for_backward(packed)     # bits/8 bytes per element; x itself is not kept
        return y.view(x.shape)

    @staticmethod
    def backward(ctx, grad_out: torch.Tensor):
        (packed,) = ctx.saved_tensors
        grad_in = fewbit_bwd(ctx.table, packed, _flat_aligned(grad_out))
        return grad_in.view(grad_out.shape), None


class _FewBitBiasFunction(torch.autograd.Function):
    """f(x + bias) with the bias add inside the forward kernel; the gradient with respect to the
    bias is the column sum of the gradient with respect to x (accumulated in binary32)."""

    @staticmethod
    def forward(ctx, x: torch.Tensor, bias: torch.Tensor, table: Table):
        if x.dtype not in (torch.float32, torch.bfloat16, torch.float16) or not x.is_cuda:
            raise TypeError("FewBitActivation needs a CUDA tensor of dtype float32, bfloat16 or float16")
        cols = bias.numel()
        xf = x.contiguous()
        if xf.data_ptr() % 32:
            xf = xf.clone()
        y, packed = fewbit_fwd_bias(table, xf.view(-1, cols), _flat_aligned(bias.to(x.dtype)))
        ctx.table, ctx.bias_dtype = table, bias.dtype
        ctx.save_for_backward(packed)
        return y.view(x.shape)

    @staticmethod
    def backward(ctx, grad_out: torch.Tensor):
        (packed,) = ctx.saved_tensors
        grad_in = fewbit_bwd(ctx.table, packed, _flat_aligned(grad_out)).view(grad_out.shape)
        grad_bias = grad_in.reshape(-1, grad_out.shape[-1]).sum(0, dtype=torch.float32).to(ctx.bias_dtype)
        return grad_in, grad_bias, None


class FewBitActivation(nn.Module):
    """Activation whose backward pass uses a ``bits``-bit piecewise-constant derivative.

    act: gelu | silu | sigmoid | tanh | elu | softplus | leaky_relu | relu | selu.
    folded: for sigmoid / tanh, quantise |x| (one more effective bit)."""

    def __init__(self, act: str = "gelu", bits: int = 3, folded: bool = False):
        super().__init__()
        self.act, self.bits, self.folded = act, int(bits), bool(folded)
        self.table = fewbit_table_create_folded(act, bits) if folded else fewbit_table_create(act, bits)

    def forward(self, x: torch.Tensor, bias: torch.Tensor | None = None) -> torch.Tensor:
        """``bias`` (optional): one value per element of the last dimension of ``x`` (a multiple of
        8), added to ``x`` inside the kernel."""
        if bias is not None:
            return _FewBitBiasFunction.apply(x, bias, self.table)
        return _FewBitFunction.apply(x, self.table)

    def extra_repr(self) -> str:
        return f"act={self.act}, bits={self.bits}, folded={self.folded}"


def fewbit_activation(x: torch.Tensor, table: Table, bias: torch.Tensor | None = None) -> torch.Tensor:
    """Functional form: ``table`` from ``fewbit_table_create``; with ``bias``, f(x + bias)."""
    if bias is not None:
        return _FewBitBiasFunction.apply(x, bias, table)
    return _FewBitFunction.apply(x, table)


def _attention_layout(t: torch.Tensor) -> torch.Tensor:
    """`t` as the library takes it: contiguous heads, strides that are multiples of 8 elements, 16-byte alignment."""
    st = t.stride()
    if st[-1] != 1 or t.data_ptr() % 16 or any(s % 8 or s <= 0 for s, n in zip(st[:-1], t.shape[:-1]) if n > 1):
        return t.clone(memory_format=torch.contiguous_format)
    return t


class _AttentionFunction(torch.autograd.Function):
    """Keeps q, k, v, the output and one number for each row and head; the probabilities are recomputed."""

    @staticmethod
    def forward(ctx, q, k, v, q_offsets, k_offsets, slopes, distance_bias, prefix_lens, q_documents, k_documents, kw):
        q, k, v = _attention_layout(q), _attention_layout(k), _attention_layout(v)
        if distance_bias is not None:
            distance_bias = distance_bias.detach().contiguous()
        given = {"q_offsets": q_offsets, "k_offsets": k_offsets, "slopes": slopes, "distance_bias": distance_bias, "prefix_lens": prefix_lens,
                 "q_documents": q_documents, "k_documents": k_documents}
        out, lse = fewbit_attention_fwd(q, k, v, **given, **kw)
        ctx.kw, ctx.names = kw, tuple(given)
        ctx.save_for_backward(q, k, v, out, lse, *given.values())        # (autograd refuses a backward pass when one has been changed)
        return out

    @staticmethod
    @once_differentiable
    def backward(ctx, grad_out):
        q, k, v, out, lse, *given = ctx.saved_tensors
        want_bias = ctx.needs_input_grad[6]
        grads = fewbit_attention_bwd(_attention_layout(grad_out), q, k, v, out, lse, bias_grad=want_bias, **dict(zip(ctx.names, given)), **ctx.kw)
        return (*grads[:3], None, None, None, grads[3] if want_bias else None, None, None, None, None)


def fewbit_attention(q: torch.Tensor, k: torch.Tensor, v: torch.Tensor, *, causal: bool = False, scale: float | None = None,
                     q_offsets: torch.Tensor | None = None, k_offsets: torch.Tensor | None = None,
                     max_q_len: int | None = None, max_k_len: int | None = None, cap: float | None = None,
                     slopes: torch.Tensor | None = None, distance_bias: torch.Tensor | None = None, prefix_lens: torch.Tensor | None = None,
                     q_documents: torch.Tensor | None = None, k_documents: torch.Tensor | None = None) -> torch.Tensor:
    """softmax(scale q k^T) v with gradients for q, k, v and ``distance_bias``; arguments as in ``fewbit_attention_fwd``.  Tensors
    whose strides the library does not take (a transposed head, an expanded batch) are copied first.  Offsets, slopes, prefixes and
    documents are kept for the backward pass as they are: a program that reuses their buffers before it gets autograd's error.  Should
    a wait inside a kernel give up (a broken device: two seconds), the results that it leaves unfinished are NaN, and
    ``fewbit_attention_timeout_count`` tells."""
    if slopes is not None and slopes.requires_grad and torch.is_grad_enabled():
        raise ValueError("slopes have no gradient here: pass ones that do not require one (detach them), or a distance_bias")
    return _AttentionFunction.apply(q, k, v, q_offsets, k_offsets, slopes, distance_bias, prefix_lens, q_documents, k_documents,
                                    {"causal": causal, "scale": scale, "max_q_len": max_q_len, "max_k_len": max_k_len, "cap": cap})


class _RelativeBiasFunction(torch.autograd.Function):
    @staticmethod
    def forward(ctx, table, max_distance, bidirectional):
        ctx.bidirectional = bidirectional
        ctx.like = table.new_empty(()), table.shape                     # type and shape alone are kept
        return fewbit_relative_bias_fwd(table.contiguous(), max_distance, bidirectional=bidirectional)

    @staticmethod
    @once_differentiable
    def backward(ctx, grad):
        like, shape = ctx.like
        return fewbit_relative_bias_bwd(grad.contiguous(), like.expand(shape), bidirectional=ctx.bidirectional), None, None


def fewbit_relative_bias(table: torch.Tensor, max_distance: int, *, bidirectional: bool = False) -> torch.Tensor:
    """A learned bias of relative positions, (buckets, heads), as the ``distance_bias`` of ``fewbit_attention``, with the table's
    gradient; arguments as in ``fewbit_relative_bias_fwd``.  One result can serve all layers that share the table."""
    return _RelativeBiasFunction.apply(table, max_distance, bidirectional)


def _contiguous_heads(t: torch.Tensor) -> torch.Tensor:
    return t if t.stride(-1) == 1 or t.shape[-1] == 1 else t.contiguous()


class _QkNormRopeFunction(torch.autograd.Function):
    """Keeps the inputs only: the norm's factor is recomputed."""

    @staticmethod
    def forward(ctx, q, k, q_weight, k_weight, cos, sin, positions, kw):
        q, k = _contiguous_heads(q), _contiguous_heads(k)
        wide = [None if w is None else w.detach().float().contiguous() for w in (q_weight, k_weight)]
        out = fewbit_qk_norm_rope_fwd(q, k, *wide, cos, sin, positions=positions, **kw)
        ctx.kw, ctx.weight_types = kw, [None if w is None else w.dtype for w in (q_weight, k_weight)]
        ctx.save_for_backward(q, k, *wide, cos, sin, positions)
        return out

    @staticmethod
    @once_differentiable
    def backward(ctx, grad_q, grad_k):
        q, k, qw, kw_, cos, sin, positions = ctx.saved_tensors
        wanted = (ctx.needs_input_grad[2] and qw is not None) or (ctx.needs_input_grad[3] and kw_ is not None)
        dq, dk, dqw, dkw = fewbit_qk_norm_rope_bwd(_contiguous_heads(grad_q), _contiguous_heads(grad_k), q, k, qw, kw_, cos, sin,
                                                   positions=positions, weight_grads=wanted, **ctx.kw)
        dws = [g.to(t) if g is not None and t is not None else None for g, t in zip((dqw, dkw), ctx.weight_types)]
        return dq, dk, dws[0], dws[1], None, None, None, None


def fewbit_qk_norm_rope(q: torch.Tensor, k: torch.Tensor, q_weight: torch.Tensor | None, k_weight: torch.Tensor | None,
                        cos: torch.Tensor | None, sin: torch.Tensor | None, *, positions: torch.Tensor | None = None,
                        eps: float = 1e-6, interleaved: bool = False):
    """RMS norm of every query and key head and the position rotation, with gradients for q, k and the weights (of any
    floating type), but none for the tables; arguments as in ``fewbit_qk_norm_rope_fwd``.  Tables and positions are kept for the
    backward pass as they are: a program that changes them before it gets autograd's error."""
    if torch.is_grad_enabled() and any(t is not None and t.requires_grad for t in (cos, sin)):
        raise ValueError("cos and sin have no gradient here: pass tables that do not require one (detach them)")
    return _QkNormRopeFunction.apply(q, k, q_weight, k_weight, cos, sin, positions, {"eps": eps, "interleaved": interleaved})


def _kept_seed(ctx, seed, *tensors):
    """Keeps the call's tensors and a seed on the device (autograd then refuses a backward pass when one has been changed)."""
    ctx.seed = None if isinstance(seed, torch.Tensor) else seed
    ctx.save_for_backward(*tensors, seed if isinstance(seed, torch.Tensor) else None)


class _DropoutFunction(torch.autograd.Function):
    """Keeps nothing but the seed."""

    @staticmethod
    def forward(ctx, x, residual, seed, p, place):
        ctx.p, ctx.place = p, place
        _kept_seed(ctx, seed)
        return fewbit_dropout_fwd(x.contiguous(), p, seed=seed, place=place, residual=None if residual is None else residual.contiguous())

    @staticmethod
    @once_differentiable
    def backward(ctx, grad):
        (seed,) = ctx.saved_tensors
        dx = fewbit_dropout_bwd(grad.contiguous(), ctx.p, seed=ctx.seed if seed is None else seed, place=ctx.place) if ctx.needs_input_grad[0] else None
        return dx, grad if ctx.needs_input_grad[1] else None, None, None, None


def fewbit_dropout(x: torch.Tensor, p: float, *, seed, place: int = 0, residual: torch.Tensor | None = None) -> torch.Tensor:
    """``residual`` + dropout of ``x`` (without it: the dropout alone) with gradients for both; arguments as in
    ``fewbit_dropout_fwd``.  Nothing is kept for the backward pass: the mask is drawn again from ``seed`` and ``place``.  A seed
    on the device that is changed before the backward pass is autograd's error.  Evaluation: p = 0."""
    return _DropoutFunction.apply(x, residual, seed, float(p), place)


class _AddRmsNormFunction(torch.autograd.Function):
    """Keeps h, which the residual stream carries on, and the weight: mask and norm's factor are computed again."""

    @staticmethod
    def forward(ctx, x, residual, weight, seed, eps, p, place):
        wide = None if weight is None else weight.detach().float().contiguous()
        y, h = fewbit_add_rms_norm_fwd(x.contiguous(), None if residual is None else residual.contiguous(), wide, eps=eps, p=p, seed=seed, place=place)
        if h.data_ptr() == x.data_ptr():
            h = h.view_as(h)                  # an input that is returned: as a tensor of its own
        ctx.kw, ctx.weight_type = {"eps": eps, "p": p, "place": place}, None if weight is None else weight.dtype
        ctx.set_materialize_grads(False)
        _kept_seed(ctx, seed, h, wide)
        return y, h

    @staticmethod
    @once_differentiable
    def backward(ctx, grad_y, grad_h):
        h, wide, seed = ctx.saved_tensors
        want_x, want_residual, want_weight = ctx.needs_input_grad[:3]
        if grad_y is None:                    # the normed result is not used: what reaches h goes on, whatever its rows hold
            grad_h = grad_h.contiguous()
            dx = grad_h
            if want_x and ctx.kw["p"] > 0.0:
                dx = fewbit_dropout_bwd(grad_h, ctx.kw["p"], seed=ctx.seed if seed is None else seed, place=ctx.kw["place"])
            return dx if want_x else None, grad_h if want_residual else None, None, None, None, None, None
        dx, dr, dw = fewbit_add_rms_norm_bwd(grad_y.contiguous(), None if grad_h is None else grad_h.contiguous(), h, wide,
                                             seed=ctx.seed if seed is None else seed, x_grad=want_x, residual_grad=want_residual,
                                             weight_grad=want_weight, **ctx.kw)
        return dx, dr, None if dw is None else dw.to(ctx.weight_type), None, None, None, None


def fewbit_add_rms_norm(x: torch.Tensor, residual: torch.Tensor | None, weight: torch.Tensor | None, *, eps: float = 1e-6,
                        p: float = 0.0, seed=0, place: int = 0):
    """h = residual + dropout(x) and its RMS norm times ``weight`` (of any floating type), with gradients for all three; returns
    (y, h), where h goes on as the next residual.  Arguments as in ``fewbit_add_rms_norm_fwd``; the backward pass keeps h alone."""
    return _AddRmsNormFunction.apply(x, residual, weight, seed, float(eps), float(p), place)
