"""Norm of query and key heads with the rotation, forward and backward, against the formulas in 64 bits; its gradients
against differences; its refusals.

Tolerances (derived, u = 2^-24): a sum of D squares in 32 bits is off by at most D u of itself, its inverse root by half of
that and 4 u; the products and the rotation add 6 u of a pair's magnitude: (D / 2 + 12) u in all, then half a step of the
type.  The backward pass adds the dot product's D u: (2 D + 30) u of the magnitudes of its terms.  A weight's gradient sums
N terms in partial sums of at most a few thousand: 4096 u of the sum of magnitudes is a wide bound."""
import ctypes

import pytest
import torch

import paper_2202_00441_b200 as fb
from paper_2202_00441_b200 import operators as ops

U = 2.0 ** -24
HALF_STEP = {torch.float32: 2.0 ** -24, torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11}


def tables(rows, r):
    f = 100.0 ** (-torch.arange(0, r, 2, device="cuda", dtype=torch.float32) / max(r, 1))
    a = torch.arange(rows, device="cuda", dtype=torch.float32)[:, None] * f
    return a.cos(), a.sin()


def rotate(x, c, s, interleaved, back=False):
    r = 2 * c.shape[-1]
    s = -s if back else s
    a, b = (x[..., 0:r:2], x[..., 1:r:2]) if interleaved else (x[..., :r // 2], x[..., r // 2:r])
    u, v = a * c - b * s, a * s + b * c
    y = x.clone()
    if interleaved:
        y[..., 0:r:2], y[..., 1:r:2] = u, v
    else:
        y[..., :r // 2], y[..., r // 2:r] = u, v
    return y


def forward(x, w, c, s, eps, interleaved):
    n = x * (x.pow(2).mean(-1, keepdim=True) + eps).rsqrt()
    return rotate(n if w is None else n * w, c, s, interleaved)


def inputs(b, n, h, hk, d, r, dtype, layout, pos, weights, seed=0):
    g = torch.Generator(device="cuda").manual_seed(seed)
    if layout == "fused":
        qkv = torch.randn(b, n, h + 2 * hk, d, generator=g, device="cuda").to(dtype)
        q, k = qkv[:, :, :h], qkv[:, :, h:h + hk]
    elif layout == "heads_first":
        q = torch.randn(b, h, n, d, generator=g, device="cuda").to(dtype).transpose(1, 2)
        k = torch.randn(b, hk, n, d, generator=g, device="cuda").to(dtype).transpose(1, 2)
    else:                                                     # a view that starts on an odd element, odd strides
        flat = torch.randn(1 + b * n * (h + hk) * (d + 1), generator=g, device="cuda").to(dtype)
        q = flat[1:1 + b * n * h * (d + 1)].view(b, n, h, d + 1)[..., :d]
        k = flat[1 + b * n * h * (d + 1):].view(b, n, hk, d + 1)[..., :d]
    w = [1 + 0.3 * torch.randn(d, generator=g, device="cuda") for _ in range(2)] if weights else [None, None]
    rows = n + 9
    c, s = tables(rows, r) if r else (None, None)
    p = None if pos is None else torch.randint(0, rows, (b, n), generator=g, device="cuda").to(pos)
    return q, k, w, c, s, p


def gathered(c, s, p, b, n, r):
    if c is None:
        z = torch.zeros(b, n, 1, 0, device="cuda", dtype=torch.float64)
        return z, z
    at = torch.arange(n, device="cuda").expand(b, n) if p is None else p.long()
    return c.double()[at].unsqueeze(2), s.double()[at].unsqueeze(2)


CASES = [
    # b, n, h, hk, d, r, dtype, interleaved, layout, positions, weights
    (1, 1, 1, 1, 2, 2, torch.float32, False, "fused", None, True),
    (2, 5, 3, 2, 64, 64, torch.float32, False, "fused", torch.int64, True),
    (2, 33, 8, 2, 128, 128, torch.bfloat16, False, "fused", None, True),
    (1, 700, 7, 1, 128, 64, torch.float16, False, "heads_first", torch.int32, True),
    (3, 17, 5, 3, 80, 40, torch.float16, True, "fused", torch.int32, True),
    (2, 19, 4, 4, 96, 96, torch.bfloat16, True, "heads_first", None, False),
    (1, 40, 9, 2, 256, 256, torch.bfloat16, False, "fused", torch.int64, True),
    (1, 11, 2, 1, 256, 128, torch.float32, True, "fused", None, True),
    (2, 13, 3, 1, 64, 20, torch.bfloat16, False, "odd", None, True),
    (2, 13, 3, 1, 64, 20, torch.bfloat16, True, "odd", torch.int32, True),
    (1, 9, 2, 2, 250, 250, torch.float32, False, "odd", None, True),
    (1, 6, 3, 0, 72, 36, torch.bfloat16, False, "fused", None, True),
    (1, 6, 0, 3, 66, 0, torch.float16, False, "fused", None, True),
    (1, 0, 2, 2, 64, 64, torch.float32, False, "fused", None, True),
    (1, 9000, 6, 2, 32, 32, torch.bfloat16, False, "fused", None, True),
    # several rounds of tokens for each CTA, chunks of 1, 2, 3 and 8 heads
    (1, 20011, 1, 2, 64, 64, torch.bfloat16, False, "fused", None, True),
    (3, 5003, 9, 3, 128, 128, torch.float16, True, "fused", torch.int32, True),
    (1, 12007, 3, 1, 128, 128, torch.float32, False, "heads_first", torch.int64, True),
]


@pytest.mark.gpu
@pytest.mark.parametrize("case", CASES, ids=lambda c: "x".join(map(str, c[:6])) + f"_{str(c[6])[6:]}_{c[8]}_{int(c[7])}")
def test_forward_and_backward_match_the_formulas(case):
    b, n, h, hk, d, r, dtype, inter, layout, pos, weights = case
    q, k, w, c, s, p = inputs(b, n, h, hk, d, r, dtype, layout, pos, weights)
    kw = dict(positions=p, eps=1e-5, interleaved=inter)
    q0, k0 = q.clone(), k.clone()
    qo, ko = fb.fewbit_qk_norm_rope_fwd(q, k, *w, c, s, **kw)
    g = torch.Generator(device="cuda").manual_seed(1)
    gq, gk = (torch.randn(x.shape, generator=g, device="cuda").to(dtype) for x in (q, k))
    dq, dk, dqw, dkw = fb.fewbit_qk_norm_rope_bwd(gq, gk, q, k, *w, c, s, **kw)
    assert torch.equal(q, q0) and torch.equal(k, k0)
    cc, ss = gathered(c, s, p, b, n, r)
    for x, wt, y, gy, dx, dw in ((q, w[0], qo, gq, dq, dqw), (k, w[1], ko, gk, dk, dkw)):
        x64 = x.double().requires_grad_()
        w64 = (torch.ones(d, device="cuda") if wt is None else wt).double().requires_grad_()
        ref = forward(x64, w64, cc, ss, 1e-5, inter)
        ref.backward(gy.double())
        with torch.no_grad():
            size = rotate((x64.abs() * (x64.pow(2).mean(-1, keepdim=True) + 1e-5).rsqrt() * w64.abs()), cc.abs(), -ss.abs(), inter)
            size = torch.maximum(size, ref.abs())              # |a c| + |b s| on the first half; the second has it anyway
            if 2 * cc.shape[-1]:
                size = size + size.flip(-1).amax(-1, keepdim=True)
            tol = (d / 2 + 12) * U * size + HALF_STEP[dtype] * 1.01 * ref.abs() + (2.0 ** -25 if dtype == torch.float16 else 0)
            assert ((y.double() - ref).abs() <= tol).all()
            rstd = (x64.pow(2).mean(-1, keepdim=True) + 1e-5).rsqrt()
            terms = (gy.double().abs().amax(-1, keepdim=True) * 1.5 * w64.abs().amax() * rstd)
            terms = terms * (1 + x64.abs() * rstd * (x64.abs() * rstd).mean(-1, keepdim=True))
            tol = (2 * d + 30) * U * terms + HALF_STEP[dtype] * 1.01 * x64.grad.abs() + (2.0 ** -25 if dtype == torch.float16 else 0)
            assert ((dx.double() - x64.grad).abs() <= tol).all()
            gr = rotate(gy.double(), cc, ss, inter, back=True)
            mags = (gr * x64 * rstd).abs().sum((0, 1, 2))
            assert ((dw.double() - w64.grad).abs() <= 4096 * U * mags + 1e-30).all()


@pytest.mark.gpu
def test_gradient_against_differences():
    """Central differences of the forward kernel in float32: step h = 2^-6 on inputs of size 1; the third-derivative term is
    about h^2, the rounding term 2^-22 / h: 3e-3 covers both."""
    q, k, w, c, s, p = inputs(1, 3, 2, 1, 16, 16, torch.float32, "fused", torch.int32, True)
    q, k = q.contiguous(), k.contiguous()
    g = torch.Generator(device="cuda").manual_seed(2)
    gq, gk = (torch.randn(x.shape, generator=g, device="cuda") for x in (q, k))
    dq, dk, dqw, _ = fb.fewbit_qk_norm_rope_bwd(gq, gk, q, k, *w, c, s, positions=p)

    def loss(q, k, w):
        a, b = fb.fewbit_qk_norm_rope_fwd(q, k, *w, c, s, positions=p)
        return float((a.double() * gq.double()).sum() + (b.double() * gk.double()).sum())

    h = 2.0 ** -6
    for t, grad, rebuild in ((q, dq, lambda x: (x, k, w)), (k, dk, lambda x: (q, x, w)), (w[0], dqw, lambda x: (q, k, [x, w[1]]))):
        for i in range(0, t.numel(), 5):
            up, dn = t.clone(), t.clone()
            up.view(-1)[i] += h
            dn.view(-1)[i] -= h
            d = (loss(*rebuild(up)) - loss(*rebuild(dn))) / (2 * h)
            assert abs(d - float(grad.view(-1)[i])) <= 3e-3 * (1 + abs(d))


@pytest.mark.gpu
def test_positions_outside_the_tables_make_nan_and_read_nothing():
    q, k, w, c, s, _ = inputs(1, 4, 2, 1, 64, 64, torch.bfloat16, "fused", None, True)
    p = torch.tensor([[0, -1, c.shape[0], c.shape[0] - 1]], device="cuda")
    qo, ko = fb.fewbit_qk_norm_rope_fwd(q, k, *w, c, s, positions=p)
    assert qo[0, [1, 2]].isnan().all() and ko[0, [1, 2]].isnan().all()
    assert qo[0, [0, 3]].isfinite().all()


@pytest.mark.gpu
@pytest.mark.parametrize("d,r", [(64, 64), (64, 32)])
def test_gradients_of_positions_outside_the_tables_are_nan(d, r):
    q, k, w, c, s, _ = inputs(1, 4, 2, 1, d, r, torch.bfloat16, "fused", None, True)
    p = torch.tensor([[0, -1, c.shape[0], c.shape[0] - 1]], device="cuda")
    gq, gk = torch.ones_like(q), torch.ones_like(k)
    dq, dk, dqw, dkw = fb.fewbit_qk_norm_rope_bwd(gq, gk, q, k, *w, c, s, positions=p)
    good = fb.fewbit_qk_norm_rope_bwd(gq[:, ::3], gk[:, ::3], q[:, ::3], k[:, ::3], *w, c, s, positions=p[:, ::3].contiguous())
    assert dq[0, [1, 2], :, :r].isnan().all() and dk[0, [1, 2], :, :r].isnan().all()
    assert torch.equal(dq[:, ::3], good[0]) and torch.equal(dk[:, ::3], good[1])
    assert dqw[:r].isnan().all() and dkw[:r].isnan().all()


@pytest.mark.gpu
def test_in_place_other_stream_and_repeatability():
    q, k, w, c, s, p = inputs(2, 50, 6, 2, 128, 128, torch.bfloat16, "fused", None, True)
    qo, ko = fb.fewbit_qk_norm_rope_fwd(q, k, *w, c, s)
    gq, gk = torch.ones_like(qo), torch.ones_like(ko)
    one = fb.fewbit_qk_norm_rope_bwd(gq, gk, q, k, *w, c, s)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    two = fb.fewbit_qk_norm_rope_bwd(gq, gk, q, k, *w, c, s, stream=side)
    torch.cuda.current_stream().wait_stream(side)
    assert all(torch.equal(a, b) for a, b in zip(one, two))
    fb.fewbit_qk_norm_rope_bwd(gq, gk, q, k, *w, c, s, out=(gq, gk), weight_grads=False)
    assert torch.equal(gq, one[0]) and torch.equal(gk, one[1])
    fb.fewbit_qk_norm_rope_fwd(q, k, *w, c, s, out=(q, k))
    assert torch.equal(q, qo) and torch.equal(k, ko)


def test_library_refusals_need_no_gpu():
    lib = fb.load_library()
    A = 1 << 20
    H = ops._Heads

    def call(tensor=H(A, 4096, 1024, 128), **kw):
        base = dict(batch=1, length=4, heads=2, kv_heads=1, head_dim=128, rotary_dim=64, table_rows=4, cos=A, sin=A, eps=1e-6, dtype=1)
        s = ops._QkShape(**(base | kw))
        r = ctypes.byref(tensor)
        one = lib.fewbit_qk_norm_rope_fwd(ctypes.byref(s), r, r, r, r, None)
        two = lib.fewbit_qk_norm_rope_bwd(ctypes.byref(s), r, r, r, r, r, r, None, None, None, 0, None)
        assert one == two
        return one

    for kw in ({"batch": -1}, {"head_dim": 63}, {"head_dim": 0}, {"rotary_dim": 3}, {"rotary_dim": 130}, {"eps": -1.0},
               {"eps": float("nan")}, {"dtype": 5}, {"cos": None}, {"table_rows": 3}, {"heads": -1}):
        assert call(**kw) == 1, kw
    assert call(head_dim=258) == 2
    assert call(batch=1 << 20, length=1 << 20, table_rows=1 << 20) == 6
    assert call(cos=A + 2) == 3 and call(positions=A + 4, positions_are_64bit=1) == 3
    assert call(H(A + 1, 4096, 1024, 128)) == 3 and call(H(None, 0, 0, 0)) == 1
    assert call(length=0) == 0
    assert lib.fewbit_qk_norm_rope_fwd(None, None, None, None, None, None) == 1
    s = ops._QkShape(batch=1, length=4, heads=2, kv_heads=1, head_dim=128, rotary_dim=64, table_rows=4, cos=A, sin=A, eps=1e-6, dtype=1)
    r = ctypes.byref(H(A, 4096, 1024, 128))
    assert lib.fewbit_qk_norm_rope_bwd(ctypes.byref(s), r, r, r, r, r, r, A, None, None, 0, None) == 1
    assert lib.fewbit_qk_norm_rope_bwd(ctypes.byref(s), r, r, r, r, r, r, A, None, A + 8, 1 << 20, None) == 3
    assert lib.fewbit_qk_norm_rope_bwd(ctypes.byref(s), r, r, r, r, r, r, A + 2, None, A, 1 << 20, None) == 3
