"""Binding of the operators next to the activation in a transformer's training step: the norm of
query and key heads with the position rotation, attention, and AdamW over many tensors.  Argument marshalling
only; the arithmetic is in include/fewbit.h."""
from __future__ import annotations

import ctypes
import importlib.util
import os
from typing import Optional, Sequence

import torch

from .binding import _check, load_library


# The C structs, for callers of the C ABI through ctypes (the functions below go through the extension module).
class _Heads(ctypes.Structure):
    _fields_ = [("data", ctypes.c_void_p), ("batch_stride", ctypes.c_int64), ("row_stride", ctypes.c_int64),
                ("head_stride", ctypes.c_int64)]


class _QkShape(ctypes.Structure):
    _fields_ = [("batch", ctypes.c_int64), ("length", ctypes.c_int64), ("heads", ctypes.c_int), ("kv_heads", ctypes.c_int),
                ("head_dim", ctypes.c_int), ("rotary_dim", ctypes.c_int), ("interleaved", ctypes.c_int),
                ("positions", ctypes.c_void_p), ("positions_are_64bit", ctypes.c_int), ("table_rows", ctypes.c_int64),
                ("cos", ctypes.c_void_p), ("sin", ctypes.c_void_p), ("q_weight", ctypes.c_void_p), ("k_weight", ctypes.c_void_p),
                ("eps", ctypes.c_float), ("dtype", ctypes.c_int)]


class _AttentionShape(ctypes.Structure):
    _fields_ = [("batch", ctypes.c_int), ("heads", ctypes.c_int), ("kv_heads", ctypes.c_int), ("head_dim", ctypes.c_int),
                ("q_len", ctypes.c_int64), ("k_len", ctypes.c_int64), ("q_rows", ctypes.c_int64), ("k_rows", ctypes.c_int64),
                ("q_offsets", ctypes.c_void_p), ("k_offsets", ctypes.c_void_p), ("causal", ctypes.c_int),
                ("scale", ctypes.c_float), ("dtype", ctypes.c_int)]


class _AdamWTensor(ctypes.Structure):
    _fields_ = [("param", ctypes.c_void_p), ("exp_avg", ctypes.c_void_p), ("exp_avg_sq", ctypes.c_void_p),
                ("exp_avg_scale", ctypes.c_void_p), ("exp_avg_sq_scale", ctypes.c_void_p), ("master", ctypes.c_void_p),
                ("n", ctypes.c_uint64)]


class _AdamWOptions(ctypes.Structure):
    _fields_ = [("lr", ctypes.c_double), ("beta1", ctypes.c_double), ("beta2", ctypes.c_double), ("eps", ctypes.c_double),
                ("weight_decay", ctypes.c_double), ("step", ctypes.c_int64), ("grad_scale_device", ctypes.c_void_p),
                ("seed", ctypes.c_uint32), ("state_bits", ctypes.c_int), ("dtype", ctypes.c_int)]


_TORCH_LIB = os.path.join(os.path.dirname(os.path.abspath(__file__)), "_fewbit_torch.so")
_module = None


def _torch_module():
    """The extension module that checks tensors, allocates outputs and calls the library (csrc/fewbit_torch.cpp)."""
    global _module
    if _module is None:
        load_library()                               # the module is linked to the same file
        if not os.path.exists(_TORCH_LIB):
            raise RuntimeError(f"{_TORCH_LIB} is missing: build it with `python -m paper_2202_00441_b200.build`")
        spec = importlib.util.spec_from_file_location("_fewbit_torch", _TORCH_LIB)
        _module = importlib.util.module_from_spec(spec)
        spec.loader.exec_module(_module)
    return _module


class _On:
    """Context of a call on `stream`: outputs are allocated for that stream, and the memory of the call's inputs is not
    handed out again before the call has read it."""

    def __init__(self, stream, *tensors):
        tensors = [t for t in tensors if t is not None]
        if any(t.device != stream.device for t in tensors):
            raise ValueError("the stream is of another device than the tensors")   # (the call would go to the current stream of theirs)
        for t in tensors:
            t.record_stream(stream)
        self.inner = torch.cuda.stream(stream)

    def __enter__(self):
        self.inner.__enter__()

    def __exit__(self, *exc):
        return self.inner.__exit__(*exc)


# ---------------------------------------------------------------------------------------------------------------
# norm of queries and keys with the position rotation
# ---------------------------------------------------------------------------------------------------------------

def fewbit_qk_norm_rope_fwd(q: torch.Tensor, k: torch.Tensor, q_weight: Optional[torch.Tensor], k_weight: Optional[torch.Tensor],
                            cos: Optional[torch.Tensor], sin: Optional[torch.Tensor], *, positions: Optional[torch.Tensor] = None,
                            eps: float = 1e-6, interleaved: bool = False, out=None, stream: Optional[torch.cuda.Stream] = None):
    """RMS norm of every head of ``q`` and ``k`` (times a weight vector), then the rotation by ``cos`` / ``sin`` at the
    token's position; returns (q_out, k_out).

    q, k: (batch, length, heads, head_dim) with any strides but contiguous heads, e.g. views of one fused projection.
    q_weight, k_weight: (head_dim,) float32 or None.  cos, sin: (rows, rotary_dim / 2) float32 tables, or None for no
    rotation; ``positions`` (batch, length) picks their rows (a position past the tables makes its heads NaN), without it
    token i has position i.  ``interleaved``: neighbouring elements are rotated with each other instead of the two
    halves.  ``out``: a pair of tensors to write to (q and k themselves are allowed, but
    no other overlap)."""
    q_out, k_out = (None, None) if out is None else out
    if stream is not None:
        with _On(stream, q, k, q_weight, k_weight, cos, sin, positions, q_out, k_out):
            return _torch_module().qk_norm_rope_fwd(q, k, q_weight, k_weight, cos, sin, positions, eps, interleaved, q_out, k_out)
    return _torch_module().qk_norm_rope_fwd(q, k, q_weight, k_weight, cos, sin, positions, eps, interleaved, q_out, k_out)


def fewbit_qk_norm_rope_bwd(grad_q_out: torch.Tensor, grad_k_out: torch.Tensor, q: torch.Tensor, k: torch.Tensor,
                            q_weight: Optional[torch.Tensor], k_weight: Optional[torch.Tensor], cos: Optional[torch.Tensor],
                            sin: Optional[torch.Tensor], *, positions: Optional[torch.Tensor] = None, eps: float = 1e-6,
                            interleaved: bool = False, weight_grads: bool = True, out=None,
                            stream: Optional[torch.cuda.Stream] = None):
    """Gradients of ``fewbit_qk_norm_rope_fwd`` from its inputs and the gradients of its outputs; returns
    (grad_q, grad_k, grad_q_weight, grad_k_weight), the last two float32 (None without ``weight_grads``)."""
    q_out, k_out = (None, None) if out is None else out
    args = (grad_q_out, grad_k_out, q, k, q_weight, k_weight, cos, sin, positions, eps, interleaved, weight_grads, q_out, k_out)
    if stream is not None:
        with _On(stream, grad_q_out, grad_k_out, q, k, q_weight, k_weight, cos, sin, positions, q_out, k_out):
            return _torch_module().qk_norm_rope_bwd(*args)
    return _torch_module().qk_norm_rope_bwd(*args)


# ---------------------------------------------------------------------------------------------------------------
# attention
# ---------------------------------------------------------------------------------------------------------------

def fewbit_attention_fwd(q: torch.Tensor, k: torch.Tensor, v: torch.Tensor, *, causal: bool = False, scale: Optional[float] = None,
                         q_offsets: Optional[torch.Tensor] = None, k_offsets: Optional[torch.Tensor] = None,
                         max_q_len: Optional[int] = None, max_k_len: Optional[int] = None,
                         stream: Optional[torch.cuda.Stream] = None):
    """softmax(scale q k^T) v for every head; returns (out, lse).

    q: (batch, q_len, heads, head_dim), k and v: (batch, k_len, kv_heads, head_dim), bfloat16 or float16, head_dim a multiple
    of 8 up to 128, any strides that are multiples of 8 with contiguous heads; query head h reads key head
    h // (heads // kv_heads).  ``causal``: row i sees keys up to i + k_len - q_len.  ``scale``: head_dim ** -0.5.
    Packed sequences: q (rows, heads, head_dim), k and v (key rows, ...), with int32 ``q_offsets`` and ``k_offsets`` on the
    device (batch + 1 values each) and the longest sequence's lengths ``max_q_len`` and ``max_k_len``.
    lse: float32 (batch, heads, q_len), or (heads, rows) when packed: the logarithm of each row's sum of exponentials,
    -inf for a row that sees no key (whose out is 0)."""
    if stream is not None:
        with _On(stream, q, k, v, q_offsets, k_offsets):
            return _torch_module().attention_fwd(q, k, v, causal, scale, q_offsets, k_offsets, max_q_len, max_k_len)
    return _torch_module().attention_fwd(q, k, v, causal, scale, q_offsets, k_offsets, max_q_len, max_k_len)


def fewbit_attention_bwd(grad_out: torch.Tensor, q: torch.Tensor, k: torch.Tensor, v: torch.Tensor, out: torch.Tensor,
                         lse: torch.Tensor, *, causal: bool = False, scale: Optional[float] = None,
                         q_offsets: Optional[torch.Tensor] = None, k_offsets: Optional[torch.Tensor] = None,
                         max_q_len: Optional[int] = None, max_k_len: Optional[int] = None,
                         stream: Optional[torch.cuda.Stream] = None):
    """Gradients (grad_q, grad_k, grad_v) of ``fewbit_attention_fwd`` from its inputs and outputs and ``grad_out``; the
    probabilities are recomputed.  The same inputs give the same bits."""
    args = (grad_out, q, k, v, out, lse, causal, scale, q_offsets, k_offsets, max_q_len, max_k_len)
    if stream is not None:
        with _On(stream, grad_out, q, k, v, out, lse, q_offsets, k_offsets):
            return _torch_module().attention_bwd(*args)
    return _torch_module().attention_bwd(*args)


def fewbit_attention_timeout_count(device=None) -> int:
    """How often a wait inside the attention kernels gave up on ``device``; 0 unless something is broken.  Synchronises."""
    device = torch.device("cuda", torch.cuda.current_device()) if device is None else torch.device(device)
    out = ctypes.c_uint64()
    with torch.cuda.device(device):
        _check(load_library().fewbit_attention_timeout_count(ctypes.byref(out)), "fewbit_attention_timeout_count")
    return int(out.value)


# ---------------------------------------------------------------------------------------------------------------
# AdamW over many tensors
# ---------------------------------------------------------------------------------------------------------------

ADAMW_BLOCK = 256


def fewbit_adamw_create(params: Sequence[torch.Tensor], exp_avgs: Sequence[torch.Tensor], exp_avg_sqs: Sequence[torch.Tensor],
                        exp_avg_scales: Optional[Sequence[torch.Tensor]] = None,
                        exp_avg_sq_scales: Optional[Sequence[torch.Tensor]] = None,
                        masters: Optional[Sequence[torch.Tensor]] = None):
    """Handle for ``fewbit_adamw_step``.  All parameters have one dtype and lie on one device; every tensor is contiguous.

    32-bit moments: float32 ``exp_avgs`` and ``exp_avg_sqs`` (zeros at the start).  8-bit moments: float8_e4m3fn codes,
    with float32 scales of ceil(n / 256) values for each tensor; ``exp_avg_sqs`` then holds the ROOT of the second
    moment (code * scale; zeros at the start).  ``masters``: float32 copies of 16-bit parameters."""
    return _torch_module().AdamWTensors(params, exp_avgs, exp_avg_sqs, exp_avg_scales, exp_avg_sq_scales, masters)


def fewbit_adamw_step(tensors, grads: Sequence[torch.Tensor], *, step: int, lr: float, betas=(0.9, 0.999),
                      eps: float = 1e-8, weight_decay: float = 0.0, seed: int = 0, grad_scale: Optional[torch.Tensor] = None,
                      stream: Optional[torch.cuda.Stream] = None) -> None:
    """One AdamW step on all parameters of ``tensors``, in place.  ``grads``: contiguous tensors of the parameters' dtype.
    ``grad_scale``: one float32 value on the device that multiplies every gradient.  ``seed``: 32 bits for the
    stochastic rounding of 8-bit moments, a new value each step (unrelated to the last one's, as a hash gives it)."""
    if stream is not None:
        with _On(stream, grad_scale, *grads, *tensors.tensors()):
            tensors.step(grads, step, lr, betas[0], betas[1], eps, weight_decay, seed & 0xFFFFFFFF, grad_scale)
    else:
        tensors.step(grads, step, lr, betas[0], betas[1], eps, weight_decay, seed & 0xFFFFFFFF, grad_scale)
