"""ctypes binding of the operators next to the activation in a transformer's training step: the norm of
query and key heads with the position rotation, attention, and AdamW over many tensors.  Argument marshalling
only; the arithmetic is in include/fewbit.h."""
from __future__ import annotations

import contextlib
import ctypes
import struct
from typing import Optional, Sequence

import torch

from .binding import _DTYPES, _check, _stream_ptr, load_library


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


# The structs of a call are packed into one buffer: a small tensor's kernel takes less time than ctypes needs to fill
# structs field by field.  Same fields in the same order, native alignment.
_HEADS = struct.Struct("@Pqqq")
_QK_SHAPE = struct.Struct("@qqiiiiiPiqPPPPfi")
_ATTENTION_SHAPE = struct.Struct("@iiiiqqqqPPifi")
for _packed, _fields in ((_HEADS, _Heads), (_QK_SHAPE, _QkShape), (_ATTENTION_SHAPE, _AttentionShape)):
    assert ctypes.sizeof(_fields) - 7 <= _packed.size <= ctypes.sizeof(_fields)   # less padding at the end
_SHAPE_ROOM = 128                                   # a shape, then the heads
_Buffer = ctypes.c_char * (_SHAPE_ROOM + 9 * _HEADS.size)


def _put_heads(buf, first: int, tensors) -> list:
    """Packs the descriptions of `tensors` ((.., length, heads, head_dim), contiguous heads) into places first, first + 1, ...
    of the buffer; returns their addresses."""
    at = _SHAPE_ROOM + first * _HEADS.size
    base, out = ctypes.addressof(buf), []
    for t in tensors:
        st = t.stride()
        if st[-1] != 1 and t.shape[-1] > 1:
            raise ValueError("the elements of one head must be contiguous")
        if len(st) == 4:
            _HEADS.pack_into(buf, at, t.data_ptr(), st[0], st[1], st[2])
        else:
            _HEADS.pack_into(buf, at, t.data_ptr(), 0, st[0], st[1])
        out.append(base + at)
        at += _HEADS.size
    return out


_get_device = getattr(torch._C, "_cuda_getDevice", None) or torch.cuda.current_device


class _On:
    """Context of a call on `device` and, when given, on `stream`: outputs are allocated for that stream, and the memory
    of the call's inputs is not handed out again before the call has read it."""

    def __init__(self, device, stream, tensors):
        self.inner = []
        if device.index != _get_device():
            self.inner.append(torch.cuda.device(device))
        if stream is not None:
            for t in tensors:
                if t is not None:
                    t.record_stream(stream)
            self.inner.append(torch.cuda.stream(stream))

    def __enter__(self):
        for c in self.inner:
            c.__enter__()

    def __exit__(self, *exc):
        for c in reversed(self.inner):
            c.__exit__(*exc)
        return False


_PLAIN = contextlib.nullcontext()


def _on(device, stream, *tensors):
    if stream is None and device.index == _get_device():
        return _PLAIN
    return _On(device, stream, tensors)


def _need(t: torch.Tensor, name: str, device, dtype=None) -> torch.Tensor:
    if t.device != device or (dtype is not None and t.dtype != dtype):
        raise ValueError(f"{name} must be a {dtype or ''} tensor on {device}")
    return t


def _pointer(t: Optional[torch.Tensor]) -> int:
    return 0 if t is None else t.data_ptr()


# ---------------------------------------------------------------------------------------------------------------
# norm of queries and keys with the position rotation
# ---------------------------------------------------------------------------------------------------------------

def _qk_shape(buf, q, k, q_weight, k_weight, cos, sin, positions, eps, interleaved):
    """Checks the inputs and packs their shape; returns their device."""
    dtype, dev = q.dtype, q.device
    if q.dim() != 4 or k.dim() != 4 or dtype not in _DTYPES or not q.is_cuda:
        raise ValueError("q and k must be (batch, length, heads, head_dim) CUDA tensors of float32, bfloat16 or float16")
    b, n, h, d = q.shape
    kb, kn, hk, kd = k.shape
    if b != kb or n != kn or d != kd or k.dtype != dtype or k.device != dev:
        raise ValueError("q and k must have one type and device, and the same batch, length and head_dim")
    for w in (q_weight, k_weight):
        if w is not None and (w.dtype != torch.float32 or w.device != dev or w.dim() != 1 or w.numel() != d or not w.is_contiguous()):
            raise ValueError("q_weight and k_weight must be contiguous float32 vectors of head_dim values on the device of q")
    rows = rot = wide = 0
    if cos is not None and sin is not None:
        if cos.dim() != 2 or cos.shape != sin.shape or not (cos.is_contiguous() and sin.is_contiguous()) or \
                cos.dtype != torch.float32 or sin.dtype != torch.float32 or cos.device != dev or sin.device != dev:
            raise ValueError("cos and sin must be contiguous float32 (rows, rotary_dim / 2) tables on the device of q")
        rows, rot = cos.shape
    elif cos is not None or sin is not None:
        raise ValueError("cos and sin come together")
    if positions is not None:
        wide = positions.dtype == torch.int64
        if positions.shape != (b, n) or not (wide or positions.dtype == torch.int32) or not positions.is_contiguous() or positions.device != dev:
            raise ValueError("positions must be a contiguous (batch, length) tensor of int32 or int64 on the device of q")
    _QK_SHAPE.pack_into(buf, 0, b, n, h, hk, d, 2 * rot, bool(interleaved), _pointer(positions), wide, rows, _pointer(cos), _pointer(sin),
                        _pointer(q_weight), _pointer(k_weight), eps, _DTYPES[dtype])
    return dev


def _two_outputs(q, k, out, dev, dtype):
    if out is None:
        return q.new_empty(q.shape), k.new_empty(k.shape)
    a, b = out
    if a.shape != q.shape or b.shape != k.shape:
        raise ValueError("out does not match q and k")
    return _need(a, "out[0]", dev, dtype), _need(b, "out[1]", dev, dtype)


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
    buf = _Buffer()
    dev = _qk_shape(buf, q, k, q_weight, k_weight, cos, sin, positions, eps, interleaved)
    with _on(dev, stream, q, k, q_weight, k_weight, cos, sin, positions):
        q_out, k_out = _two_outputs(q, k, out, dev, q.dtype)
        hs = _put_heads(buf, 0, (q, k, q_out, k_out))
        _check(load_library().fewbit_qk_norm_rope_fwd(ctypes.addressof(buf), *hs, _stream_ptr(stream, dev)), "fewbit_qk_norm_rope_fwd")
    return q_out, k_out


def fewbit_qk_norm_rope_bwd(grad_q_out: torch.Tensor, grad_k_out: torch.Tensor, q: torch.Tensor, k: torch.Tensor,
                            q_weight: Optional[torch.Tensor], k_weight: Optional[torch.Tensor], cos: Optional[torch.Tensor],
                            sin: Optional[torch.Tensor], *, positions: Optional[torch.Tensor] = None, eps: float = 1e-6,
                            interleaved: bool = False, weight_grads: bool = True, out=None,
                            stream: Optional[torch.cuda.Stream] = None):
    """Gradients of ``fewbit_qk_norm_rope_fwd`` from its inputs and the gradients of its outputs; returns
    (grad_q, grad_k, grad_q_weight, grad_k_weight), the last two float32 (None without ``weight_grads``)."""
    buf = _Buffer()
    dev = _qk_shape(buf, q, k, q_weight, k_weight, cos, sin, positions, eps, interleaved)
    if grad_q_out.shape != q.shape or grad_k_out.shape != k.shape:
        raise ValueError("the gradients do not match q and k")
    _need(grad_q_out, "grad_q_out", dev, q.dtype), _need(grad_k_out, "grad_k_out", dev, q.dtype)
    lib, base = load_library(), ctypes.addressof(buf)
    with _on(dev, stream, grad_q_out, grad_k_out, q, k, q_weight, k_weight, cos, sin, positions):
        grad_q, grad_k = _two_outputs(q, k, out, dev, q.dtype)
        grad_qw = grad_kw = ws = None
        ws_bytes = 0
        if weight_grads:
            grad_qw = torch.empty(q.shape[3], dtype=torch.float32, device=dev)
            grad_kw = torch.empty(q.shape[3], dtype=torch.float32, device=dev)
            ws_bytes = lib.fewbit_qk_norm_rope_workspace_bytes(base)
            ws = torch.empty(ws_bytes, dtype=torch.uint8, device=dev)
        hs = _put_heads(buf, 0, (grad_q_out, grad_k_out, q, k, grad_q, grad_k))
        _check(lib.fewbit_qk_norm_rope_bwd(base, *hs, _pointer(grad_qw), _pointer(grad_kw), _pointer(ws), ws_bytes, _stream_ptr(stream, dev)),
               "fewbit_qk_norm_rope_bwd")
    return grad_q, grad_k, grad_qw, grad_kw


# ---------------------------------------------------------------------------------------------------------------
# attention
# ---------------------------------------------------------------------------------------------------------------

def _attention_shape(buf, q, k, v, causal, scale, q_offsets, k_offsets, max_q_len, max_k_len):
    """Checks the inputs and packs their shape; returns their device and the shape of lse."""
    dtype, dev = q.dtype, q.device
    if (dtype != torch.bfloat16 and dtype != torch.float16) or not q.is_cuda:
        raise ValueError("attention takes bfloat16 or float16 CUDA tensors")
    if k.dtype != dtype or v.dtype != dtype or k.device != dev or v.device != dev or k.shape != v.shape:
        raise ValueError("q, k and v must have one type and device, k and v one shape")
    if q_offsets is None:
        if k_offsets is not None or max_q_len is not None or max_k_len is not None:
            raise ValueError("packed sequences need q_offsets, k_offsets, max_q_len and max_k_len, others none of them")
        if q.dim() != 4 or k.dim() != 4:
            raise ValueError("q, k and v must be (batch, length, heads, head_dim) tensors")
        b, n, h, d = q.shape
        kb, m, hk, kd = k.shape
        if kb != b or kd != d:
            raise ValueError("q, k and v must have the same batch and head_dim")
        _ATTENTION_SHAPE.pack_into(buf, 0, b, h, hk, d, n, m, 0, 0, 0, 0, bool(causal), d ** -0.5 if scale is None else scale, _DTYPES[dtype])
        return dev, (b, h, n)
    if k_offsets is None or max_q_len is None or max_k_len is None:
        raise ValueError("packed sequences need q_offsets, k_offsets, max_q_len and max_k_len, others none of them")
    if q.dim() != 3 or k.dim() != 3 or k.shape[2] != q.shape[2]:
        raise ValueError("packed sequences are (rows, heads, head_dim) tensors")
    for o in (q_offsets, k_offsets):
        if o.dtype != torch.int32 or o.device != dev or o.dim() != 1 or o.numel() < 1 or o.numel() != q_offsets.numel() or not o.is_contiguous():
            raise ValueError("q_offsets and k_offsets must be contiguous vectors of batch + 1 int32 values on the device of q")
    n, h, d = q.shape
    m, hk, _ = k.shape
    _ATTENTION_SHAPE.pack_into(buf, 0, q_offsets.numel() - 1, h, hk, d, min(max_q_len, n), min(max_k_len, m), n, m, q_offsets.data_ptr(),
                               k_offsets.data_ptr(), bool(causal), d ** -0.5 if scale is None else scale, _DTYPES[dtype])
    return dev, (h, n)


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
    buf = _Buffer()
    dev, stats = _attention_shape(buf, q, k, v, causal, scale, q_offsets, k_offsets, max_q_len, max_k_len)
    with _on(dev, stream, q, k, v, q_offsets, k_offsets):
        out, lse = q.new_empty(q.shape), torch.empty(stats, dtype=torch.float32, device=dev)
        hs = _put_heads(buf, 0, (q, k, v, out))
        _check(load_library().fewbit_attention_fwd(ctypes.addressof(buf), *hs, lse.data_ptr(), _stream_ptr(stream, dev)), "fewbit_attention_fwd")
    return out, lse


def fewbit_attention_bwd(grad_out: torch.Tensor, q: torch.Tensor, k: torch.Tensor, v: torch.Tensor, out: torch.Tensor,
                         lse: torch.Tensor, *, causal: bool = False, scale: Optional[float] = None,
                         q_offsets: Optional[torch.Tensor] = None, k_offsets: Optional[torch.Tensor] = None,
                         max_q_len: Optional[int] = None, max_k_len: Optional[int] = None,
                         stream: Optional[torch.cuda.Stream] = None):
    """Gradients (grad_q, grad_k, grad_v) of ``fewbit_attention_fwd`` from its inputs and outputs and ``grad_out``; the
    probabilities are recomputed.  The same inputs give the same bits."""
    buf = _Buffer()
    dev, stats = _attention_shape(buf, q, k, v, causal, scale, q_offsets, k_offsets, max_q_len, max_k_len)
    if grad_out.shape != q.shape or out.shape != q.shape or lse.shape != stats or not lse.is_contiguous():
        raise ValueError("grad_out, out and lse must have the shapes that the forward pass gives")
    _need(grad_out, "grad_out", dev, q.dtype), _need(out, "out", dev, q.dtype), _need(lse, "lse", dev, torch.float32)
    lib, base = load_library(), ctypes.addressof(buf)
    with _on(dev, stream, grad_out, q, k, v, out, lse, q_offsets, k_offsets):
        grads = q.new_empty(q.shape), k.new_empty(k.shape), v.new_empty(v.shape)
        ws_bytes = lib.fewbit_attention_workspace_bytes(base)
        ws = torch.empty(ws_bytes, dtype=torch.uint8, device=dev)
        hs = _put_heads(buf, 0, (grad_out, q, k, v, out, *grads))
        _check(lib.fewbit_attention_bwd(base, *hs[:5], lse.data_ptr(), *hs[5:], ws.data_ptr(), ws_bytes, _stream_ptr(stream, dev)),
               "fewbit_attention_bwd")
    return grads


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
    with _on(device, stream, grad_scale, *grads, *(tensors.tensors() if stream is not None else ())):
        _check(load_library().fewbit_adamw_step(tensors._descs, into, n, ctypes.byref(o), _stream_ptr(stream, device)),
               "fewbit_adamw_step")
