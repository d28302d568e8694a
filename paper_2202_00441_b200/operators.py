"""ctypes binding of the operators next to the activation in a transformer's training step: the norm of
query and key heads with the position rotation, attention, and AdamW over many tensors.  Argument marshalling
only; the arithmetic is in include/fewbit.h."""
from __future__ import annotations

import contextlib
import ctypes
from typing import Optional, Sequence

import torch

from .binding import _DTYPES, _check, _current, _stream_ptr, load_library


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


_NO_STREAM = contextlib.nullcontext()


def _on(stream: Optional[torch.cuda.Stream], *tensors):
    """Context in which outputs of a call on `stream` are allocated: they belong to that stream, and the memory of
    the call's inputs is not handed out again before the call has read it."""
    if stream is None:
        return _NO_STREAM
    for t in tensors:
        if t is not None:
            t.record_stream(stream)
    return torch.cuda.stream(stream)


def _need(t: torch.Tensor, name: str, device, dtype=None) -> torch.Tensor:
    if not t.is_cuda or t.device != device or (dtype is not None and t.dtype != dtype):
        raise ValueError(f"{name} must be a {dtype or ''} CUDA tensor on {device}")
    return t


def _heads(t: torch.Tensor, name: str) -> _Heads:
    if t.shape[-1] > 1 and t.stride(-1) != 1:
        raise ValueError(f"the elements of one head of {name} must be contiguous")
    if t.dim() == 4:
        return _Heads(t.data_ptr(), t.stride(0), t.stride(1), t.stride(2))
    return _Heads(t.data_ptr(), 0, t.stride(0), t.stride(1))


# ---------------------------------------------------------------------------------------------------------------
# norm of queries and keys with the position rotation
# ---------------------------------------------------------------------------------------------------------------

def _qk_shape(q, k, q_weight, k_weight, cos, sin, positions, eps, interleaved) -> _QkShape:
    if q.dim() != 4 or k.dim() != 4 or q.shape[:2] != k.shape[:2] or q.shape[3] != k.shape[3] or q.dtype not in _DTYPES:
        raise ValueError("q and k must be (batch, length, heads, head_dim) tensors of one float32, bfloat16 or float16 type, "
                         "with the same batch, length and head_dim")
    dev = q.device
    _need(q, "q", dev), _need(k, "k", dev, q.dtype)
    b, n, h, d = q.shape
    for w, name in ((q_weight, "q_weight"), (k_weight, "k_weight")):
        if w is not None and (_need(w, name, dev, torch.float32).shape != (d,) or not w.is_contiguous()):
            raise ValueError(f"{name} must be a contiguous vector of head_dim values")
    s = _QkShape(b, n, h, k.shape[2], d, 0, int(bool(interleaved)), None, 0, 0, None, None,
                 None if q_weight is None else q_weight.data_ptr(), None if k_weight is None else k_weight.data_ptr(),
                 float(eps), _DTYPES[q.dtype])
    if (cos is None) != (sin is None):
        raise ValueError("cos and sin come together")
    if cos is not None:
        if cos.dim() != 2 or cos.shape != sin.shape or not (cos.is_contiguous() and sin.is_contiguous()):
            raise ValueError("cos and sin must be contiguous (rows, rotary_dim / 2) tables")
        _need(cos, "cos", dev, torch.float32), _need(sin, "sin", dev, torch.float32)
        s.table_rows, s.rotary_dim, s.cos, s.sin = cos.shape[0], 2 * cos.shape[1], cos.data_ptr(), sin.data_ptr()
    if positions is not None:
        if positions.shape != (b, n) or positions.dtype not in (torch.int32, torch.int64) or not positions.is_contiguous():
            raise ValueError("positions must be a contiguous (batch, length) tensor of int32 or int64")
        _need(positions, "positions", dev)
        s.positions, s.positions_are_64bit = positions.data_ptr(), int(positions.dtype == torch.int64)
    return s


def fewbit_qk_norm_rope_fwd(q: torch.Tensor, k: torch.Tensor, q_weight: Optional[torch.Tensor], k_weight: Optional[torch.Tensor],
                            cos: Optional[torch.Tensor], sin: Optional[torch.Tensor], *, positions: Optional[torch.Tensor] = None,
                            eps: float = 1e-6, interleaved: bool = False, out=None, stream: Optional[torch.cuda.Stream] = None):
    """RMS norm of every head of ``q`` and ``k`` (times a weight vector), then the rotation by ``cos`` / ``sin`` at the
    token's position; returns (q_out, k_out).

    q, k: (batch, length, heads, head_dim) with any strides but contiguous heads, e.g. views of one fused projection.
    q_weight, k_weight: (head_dim,) float32 or None.  cos, sin: (rows, rotary_dim / 2) float32 tables, or None for no
    rotation; ``positions`` (batch, length) picks their rows (a position past the tables makes its heads NaN), without it
    token i has position i.  ``interleaved``: neighbouring elements are rotated with each other instead of the two
    halves.  ``out``: a pair of tensors to write to (q and k themselves are allowed)."""
    s = _qk_shape(q, k, q_weight, k_weight, cos, sin, positions, eps, interleaved)
    with _current(q.device), _on(stream, q, k, q_weight, k_weight, cos, sin, positions):
        q_out, k_out = out if out is not None else (torch.empty(q.shape, dtype=q.dtype, device=q.device),
                                                    torch.empty(k.shape, dtype=k.dtype, device=k.device))
        if q_out.shape != q.shape or k_out.shape != k.shape:
            raise ValueError("out does not match q and k")
        _need(q_out, "q_out", q.device, q.dtype), _need(k_out, "k_out", q.device, q.dtype)
        hs = [_heads(t, name) for t, name in ((q, "q"), (k, "k"), (q_out, "q_out"), (k_out, "k_out"))]
        _check(load_library().fewbit_qk_norm_rope_fwd(ctypes.byref(s), *map(ctypes.byref, hs), _stream_ptr(stream, q.device)),
               "fewbit_qk_norm_rope_fwd")
    return q_out, k_out


def fewbit_qk_norm_rope_bwd(grad_q_out: torch.Tensor, grad_k_out: torch.Tensor, q: torch.Tensor, k: torch.Tensor,
                            q_weight: Optional[torch.Tensor], k_weight: Optional[torch.Tensor], cos: Optional[torch.Tensor],
                            sin: Optional[torch.Tensor], *, positions: Optional[torch.Tensor] = None, eps: float = 1e-6,
                            interleaved: bool = False, weight_grads: bool = True, out=None,
                            stream: Optional[torch.cuda.Stream] = None):
    """Gradients of ``fewbit_qk_norm_rope_fwd`` from its inputs and the gradients of its outputs; returns
    (grad_q, grad_k, grad_q_weight, grad_k_weight), the last two float32 (None without ``weight_grads``)."""
    s = _qk_shape(q, k, q_weight, k_weight, cos, sin, positions, eps, interleaved)
    if grad_q_out.shape != q.shape or grad_k_out.shape != k.shape:
        raise ValueError("the gradients do not match q and k")
    dev = q.device
    _need(grad_q_out, "grad_q_out", dev, q.dtype), _need(grad_k_out, "grad_k_out", dev, q.dtype)
    lib = load_library()
    with _current(dev), _on(stream, grad_q_out, grad_k_out, q, k, q_weight, k_weight, cos, sin, positions):
        grad_q, grad_k = out if out is not None else (torch.empty(q.shape, dtype=q.dtype, device=dev),
                                                      torch.empty(k.shape, dtype=k.dtype, device=dev))
        if grad_q.shape != q.shape or grad_k.shape != k.shape:
            raise ValueError("out does not match q and k")
        _need(grad_q, "grad_q", dev, q.dtype), _need(grad_k, "grad_k", dev, q.dtype)
        dw, dw_ptr, ws, ws_bytes = (None, None), (None, None), None, 0
        if weight_grads:
            both = torch.empty(2, q.shape[-1], dtype=torch.float32, device=dev)
            dw = (both[0], both[1])
            dw_ptr = (both.data_ptr(), both.data_ptr() + 4 * q.shape[-1])
            ws_bytes = lib.fewbit_qk_norm_rope_workspace_bytes(ctypes.byref(s))
            ws = torch.empty(ws_bytes, dtype=torch.uint8, device=dev)
        hs = [_heads(t, name) for t, name in ((grad_q_out, "grad_q_out"), (grad_k_out, "grad_k_out"), (q, "q"), (k, "k"),
                                              (grad_q, "grad_q"), (grad_k, "grad_k"))]
        _check(lib.fewbit_qk_norm_rope_bwd(ctypes.byref(s), *map(ctypes.byref, hs), *dw_ptr, None if ws is None else ws.data_ptr(),
                                           ws_bytes, _stream_ptr(stream, dev)), "fewbit_qk_norm_rope_bwd")
    return grad_q, grad_k, dw[0], dw[1]


# ---------------------------------------------------------------------------------------------------------------
# attention
# ---------------------------------------------------------------------------------------------------------------

def _attention_shape(q, k, v, causal, scale, q_offsets, k_offsets, max_q_len, max_k_len) -> _AttentionShape:
    packed = q_offsets is not None
    if packed != (k_offsets is not None) or packed != (max_q_len is not None) or packed != (max_k_len is not None):
        raise ValueError("packed sequences need q_offsets, k_offsets, max_q_len and max_k_len, others none of them")
    dims = 3 if packed else 4
    if q.dim() != dims or k.dim() != dims or k.shape != v.shape or q.shape[-1] != k.shape[-1] or (not packed and q.shape[0] != k.shape[0]):
        raise ValueError("q, k and v must be (batch, length, heads, head_dim) tensors, or (rows, heads, head_dim) for packed "
                         "sequences; k and v of one shape, head_dim the same for all")
    dev = q.device
    if q.dtype not in (torch.bfloat16, torch.float16):
        raise ValueError("attention takes bfloat16 or float16 tensors")
    _need(q, "q", dev), _need(k, "k", dev, q.dtype), _need(v, "v", dev, q.dtype)
    h, hk, d = q.shape[-2], k.shape[-2], q.shape[-1]
    scale = d ** -0.5 if scale is None else scale
    if not packed:
        return _AttentionShape(q.shape[0], h, hk, d, q.shape[1], k.shape[1], 0, 0, None, None, int(bool(causal)), scale, _DTYPES[q.dtype])
    for o, name in ((q_offsets, "q_offsets"), (k_offsets, "k_offsets")):
        if _need(o, name, dev, torch.int32).dim() != 1 or o.numel() < 1 or o.numel() != q_offsets.numel() or not o.is_contiguous():
            raise ValueError(f"{name} must be a contiguous vector of batch + 1 int32 values")
    return _AttentionShape(q_offsets.numel() - 1, h, hk, d, min(max_q_len, q.shape[0]), min(max_k_len, k.shape[0]), q.shape[0], k.shape[0],
                           q_offsets.data_ptr(), k_offsets.data_ptr(), int(bool(causal)), scale, _DTYPES[q.dtype])


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
    s = _attention_shape(q, k, v, causal, scale, q_offsets, k_offsets, max_q_len, max_k_len)
    packed = q_offsets is not None
    with _current(q.device), _on(stream, q, k, v, q_offsets, k_offsets):
        # rows of no sequence are not written by the library: they are zero here
        out = (torch.zeros if packed else torch.empty)(q.shape, dtype=q.dtype, device=q.device)
        lse = torch.full((q.shape[1], q.shape[0]), -float("inf"), dtype=torch.float32, device=q.device) if packed else \
            torch.empty((q.shape[0], q.shape[2], q.shape[1]), dtype=torch.float32, device=q.device)
        hs = [_heads(t, name) for t, name in ((q, "q"), (k, "k"), (v, "v"), (out, "out"))]
        _check(load_library().fewbit_attention_fwd(ctypes.byref(s), *map(ctypes.byref, hs), lse.data_ptr(), _stream_ptr(stream, q.device)),
               "fewbit_attention_fwd")
    return out, lse


def fewbit_attention_bwd(grad_out: torch.Tensor, q: torch.Tensor, k: torch.Tensor, v: torch.Tensor, out: torch.Tensor,
                         lse: torch.Tensor, *, causal: bool = False, scale: Optional[float] = None,
                         q_offsets: Optional[torch.Tensor] = None, k_offsets: Optional[torch.Tensor] = None,
                         max_q_len: Optional[int] = None, max_k_len: Optional[int] = None,
                         stream: Optional[torch.cuda.Stream] = None):
    """Gradients (grad_q, grad_k, grad_v) of ``fewbit_attention_fwd`` from its inputs and outputs and ``grad_out``; the
    probabilities are recomputed.  The same inputs give the same bits."""
    s = _attention_shape(q, k, v, causal, scale, q_offsets, k_offsets, max_q_len, max_k_len)
    packed = q_offsets is not None
    dev = q.device
    stats = (q.shape[1], q.shape[0]) if packed else (q.shape[0], q.shape[2], q.shape[1])
    if grad_out.shape != q.shape or out.shape != q.shape or lse.shape != stats or not lse.is_contiguous():
        raise ValueError("grad_out, out and lse must have the shapes that the forward pass gives")
    _need(grad_out, "grad_out", dev, q.dtype), _need(out, "out", dev, q.dtype), _need(lse, "lse", dev, torch.float32)
    lib = load_library()
    with _current(dev), _on(stream, grad_out, q, k, v, out, lse, q_offsets, k_offsets):
        new = torch.zeros if packed else torch.empty
        grads = [new(t.shape, dtype=q.dtype, device=dev) for t in (q, k, v)]
        ws_bytes = 4 * lse.numel()
        ws = torch.empty(lse.numel(), dtype=torch.float32, device=dev)
        hs = [_heads(t, name) for t, name in ((grad_out, "grad_out"), (q, "q"), (k, "k"), (v, "v"), (out, "out"))]
        gs = [_heads(t, name) for t, name in zip(grads, ("grad_q", "grad_k", "grad_v"))]
        _check(lib.fewbit_attention_bwd(ctypes.byref(s), *map(ctypes.byref, hs), lse.data_ptr(), *map(ctypes.byref, gs), ws.data_ptr(),
                                        ws_bytes, _stream_ptr(stream, dev)), "fewbit_attention_bwd")
    return tuple(grads)


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


class AdamWTensors:
    """The parameters and moments of ``fewbit_adamw_step``, as the library wants them: made once, used every step.
    Keeps the tensors alive; they are updated in place."""

    def __init__(self, params, exp_avgs, exp_avg_sqs, exp_avg_scales, exp_avg_sq_scales, masters):
        n = len(params)
        lists = [exp_avgs, exp_avg_sqs, exp_avg_scales, exp_avg_sq_scales, masters]
        if n == 0 or any(x is not None and len(x) != n for x in lists):
            raise ValueError("every list must have one tensor for each parameter, and there must be one")
        if (exp_avg_scales is None) != (exp_avg_sq_scales is None):
            raise ValueError("the scales of both moments come together")
        self.bits = 32 if exp_avg_scales is None else 8
        self.dtype, self.device = params[0].dtype, params[0].device
        if self.dtype not in _DTYPES:
            raise ValueError("parameters must be float32, bfloat16 or float16")
        if masters is not None and self.dtype == torch.float32:
            raise ValueError("float32 parameters need no master copy")
        state = torch.float32 if self.bits == 32 else torch.float8_e4m3fn

        def pointer(x, i, dtype, numel, name):
            if x is None:
                return None
            t = x[i]
            if t.device != self.device or not t.is_cuda or t.dtype != dtype or t.numel() != numel or not t.is_contiguous():
                raise ValueError(f"{name}[{i}] must be a contiguous {dtype} CUDA tensor of {numel} elements on {self.device}")
            return t.data_ptr()

        self._descs = (_AdamWTensor * n)()
        self.numels = [p.numel() for p in params]
        for i, numel in enumerate(self.numels):
            blocks = -(-numel // ADAMW_BLOCK)
            self._descs[i] = _AdamWTensor(pointer(params, i, self.dtype, numel, "params"),
                                          pointer(exp_avgs, i, state, numel, "exp_avgs"),
                                          pointer(exp_avg_sqs, i, state, numel, "exp_avg_sqs"),
                                          pointer(exp_avg_scales, i, torch.float32, blocks, "exp_avg_scales"),
                                          pointer(exp_avg_sq_scales, i, torch.float32, blocks, "exp_avg_sq_scales"),
                                          pointer(masters, i, torch.float32, numel, "masters"), numel)
        self._keep = [params] + lists
        self._grads = (ctypes.c_void_p * n)()

    def __len__(self):
        return len(self.numels)

    def tensors(self):
        return [t for x in self._keep if x is not None for t in x]


def fewbit_adamw_create(params: Sequence[torch.Tensor], exp_avgs: Sequence[torch.Tensor], exp_avg_sqs: Sequence[torch.Tensor],
                        exp_avg_scales: Optional[Sequence[torch.Tensor]] = None,
                        exp_avg_sq_scales: Optional[Sequence[torch.Tensor]] = None,
                        masters: Optional[Sequence[torch.Tensor]] = None) -> AdamWTensors:
    """Handle for ``fewbit_adamw_step``.  All parameters have one dtype and lie on one device; every tensor is contiguous.

    32-bit moments: float32 ``exp_avgs`` and ``exp_avg_sqs`` (zeros at the start).  8-bit moments: float8_e4m3fn codes,
    with float32 scales of ceil(n / 256) values for each tensor; ``exp_avg_sqs`` then holds the ROOT of the second
    moment (code * scale; zeros at the start).  ``masters``: float32 copies of 16-bit parameters."""
    return AdamWTensors(list(params), list(exp_avgs), list(exp_avg_sqs), None if exp_avg_scales is None else list(exp_avg_scales),
                        None if exp_avg_sq_scales is None else list(exp_avg_sq_scales), None if masters is None else list(masters))


def fewbit_adamw_step(tensors: AdamWTensors, grads: Sequence[torch.Tensor], *, step: int, lr: float, betas=(0.9, 0.999),
                      eps: float = 1e-8, weight_decay: float = 0.0, seed: int = 0, grad_scale: Optional[torch.Tensor] = None,
                      stream: Optional[torch.cuda.Stream] = None) -> None:
    """One AdamW step on all parameters of ``tensors``, in place.  ``grads``: contiguous tensors of the parameters' dtype.
    ``grad_scale``: one float32 value on the device that multiplies every gradient.  ``seed``: 32 bits for the
    stochastic rounding of 8-bit moments, a new value each step."""
    n, dtype, device, into = len(tensors), tensors.dtype, tensors.device, tensors._grads
    if len(grads) != n:
        raise ValueError("one gradient for each parameter is needed")
    for i, (g, numel) in enumerate(zip(grads, tensors.numels)):
        if g.dtype != dtype or g.device != device or g.numel() != numel or not g.is_contiguous():
            raise ValueError(f"grads[{i}] must be a contiguous {dtype} tensor of {numel} elements on {device}")
        into[i] = g.data_ptr()
    if grad_scale is not None and _need(grad_scale, "grad_scale", device, torch.float32).numel() != 1:
        raise ValueError("grad_scale must be one value")
    o = _AdamWOptions(lr, betas[0], betas[1], eps, weight_decay, step, None if grad_scale is None else grad_scale.data_ptr(),
                      seed & 0xFFFFFFFF, tensors.bits, _DTYPES[dtype])
    if stream is not None:
        _on(stream, grad_scale, *grads, *tensors.tensors())
    with _current(device):
        _check(load_library().fewbit_adamw_step(tensors._descs, into, n, ctypes.byref(o), _stream_ptr(stream, device)),
               "fewbit_adamw_step")
