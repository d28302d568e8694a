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
from .operators import fewbit_attention_bwd, fewbit_attention_fwd, fewbit_qk_norm_rope_bwd, fewbit_qk_norm_rope_fwd


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
    def forward(ctx, q, k, v, q_offsets, k_offsets, kw):
        q, k, v = _attention_layout(q), _attention_layout(k), _attention_layout(v)
        out, lse = fewbit_attention_fwd(q, k, v, q_offsets=q_offsets, k_offsets=k_offsets, **kw)
        ctx.kw = kw
        ctx.save_for_backward(q, k, v, out, lse, q_offsets, k_offsets)   # (autograd refuses a backward pass when one has been changed)
        return out

    @staticmethod
    @once_differentiable
    def backward(ctx, grad_out):
        q, k, v, out, lse, q_offsets, k_offsets = ctx.saved_tensors
        return (*fewbit_attention_bwd(_attention_layout(grad_out), q, k, v, out, lse, q_offsets=q_offsets, k_offsets=k_offsets, **ctx.kw),
                None, None, None)


def fewbit_attention(q: torch.Tensor, k: torch.Tensor, v: torch.Tensor, *, causal: bool = False, scale: float | None = None,
                     q_offsets: torch.Tensor | None = None, k_offsets: torch.Tensor | None = None,
                     max_q_len: int | None = None, max_k_len: int | None = None) -> torch.Tensor:
    """softmax(scale q k^T) v with gradients; arguments as in ``fewbit_attention_fwd``.  Tensors whose strides the library
    does not take (a transposed head, an expanded batch) are copied first.  The offsets are kept for the backward pass as they
    are: a program that reuses their buffer before it gets autograd's error.  Should a wait inside a kernel give up (a broken device:
    two seconds), the results that it leaves unfinished are NaN, and ``fewbit_attention_timeout_count`` tells."""
    return _AttentionFunction.apply(q, k, v, q_offsets, k_offsets, {"causal": causal, "scale": scale, "max_q_len": max_q_len, "max_k_len": max_k_len})


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
