"""Attention, forward and backward, against the formulas in 64 bits; gradients against differences; refusals.

Tolerances (derived).  e = half a step of the 16-bit type (2^-8 / 2^-11).  The products have 32-bit sums; what is rounded to
16 bits is P, dS and the results.
 out  = sum P v: each P is off by e P: |err| <= e sum P |v| + e |out| + 32-bit terms.
 dv   = sum P dO: e sum P |dO| + e |dv| the same way; P also carries lse's and the exponential's error, below 2^-16 P here.
 delta uses the rounded out: off by e |dO| . |out| per row; dS is off by P (that) + e |dS|; dq = scale sum dS k and
 dk = scale sum dS q sum those magnitudes, and are rounded themselves.
binary16 has an absolute step of 2^-25 as well, which counts once for every P and dS that falls below its normal range.
Each bound is multiplied by 1.05 for the 32-bit sums (at most 4096 terms: 2^-12 of the magnitudes)."""
import ctypes
import math

import pytest
import torch

import paper_2202_00441_b200 as fb
from paper_2202_00441_b200 import operators as ops

E = {torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11}
TINY = {torch.bfloat16: 0.0, torch.float16: 2.0 ** -25}


def reference(q, k, v, g, causal, scale):
    """One sequence: q, g (n, h, d), k, v (m, hk, d), 64 bits.  Values and the magnitudes that the tolerances need."""
    n, h, d = q.shape
    m, hk = k.shape[:2]
    q, g = (x.transpose(0, 1) for x in (q, g))
    k, v = (x.transpose(0, 1).repeat_interleave(h // hk, 0) for x in (k, v))
    s = scale * q @ k.transpose(1, 2)
    if causal:
        s = s.masked_fill(torch.ones(n, m, dtype=torch.bool, device=q.device).triu(1 + m - n), -math.inf)
    lse = torch.logsumexp(s, -1) if m else torch.full((h, n), -math.inf, dtype=torch.float64, device=q.device)
    p = torch.where(s == -math.inf, 0.0, (s - torch.where(lse == -math.inf, 0.0, lse)[..., None]).exp())
    out = p @ v
    dp = g @ v.transpose(1, 2)
    delta = (g * out).sum(-1, keepdim=True)
    ds = p * (dp - delta)
    seen = (s > -math.inf).double()

    def shared(x):
        return x.view(hk, h // hk, *x.shape[1:]).sum(1)

    r = {"out": out, "lse": lse, "dq": scale * ds @ k, "dk": shared(scale * ds.transpose(1, 2) @ q), "dv": shared(p.transpose(1, 2) @ g)}
    off_delta = (g.abs() * out.abs()).sum(-1, keepdim=True)
    ds_err = lambda e, t: e * (ds.abs() + p * off_delta + p * e * (g.abs() @ v.abs().transpose(1, 2))) + (t + p * t * g.abs().sum(-1, keepdim=True)) * seen  # noqa: E731
    tol = {
        "out": lambda e, t: (e * p + t * seen) @ v.abs() + e * out.abs() + t,
        "dv": lambda e, t: shared((e * p + t * seen).transpose(1, 2) @ g.abs()) + e * r["dv"].abs() + t,
        "dq": lambda e, t: scale * ds_err(e, t) @ k.abs() + e * r["dq"].abs() + t,
        "dk": lambda e, t: shared(scale * ds_err(e, t).transpose(1, 2) @ q.abs()) + e * r["dk"].abs() + t,
    }
    return r, tol


def compare(q, k, v, g, got, causal, scale):
    """got: out (n, h, d), lse (h, n), dq, dk, dv of one sequence."""
    dtype = q.dtype
    r, tol = reference(*(x.double() for x in (q, k, v, g)), causal, scale)
    assert torch.equal(got["lse"].double() == -math.inf, r["lse"] == -math.inf)
    fin = r["lse"] > -math.inf
    assert ((got["lse"].double() - r["lse"])[fin].abs() <= 2.0 ** -16 * (1 + r["lse"][fin].abs())).all()
    for name in ("out", "dq", "dk", "dv"):
        if name not in got or not got[name].numel():
            continue
        bound = 1.05 * tol[name](E[dtype], TINY[dtype]).transpose(0, 1) + 1e-30
        err = (got[name].double() - r[name].transpose(0, 1)).abs()
        assert (err <= bound).all(), (name, float((err / bound).max()), float(err.max()))


def make(b, n, m, h, hk, d, dtype, layout="plain", seed=0, size=1.0):
    gen = torch.Generator(device="cuda").manual_seed(seed)

    def new(*shape):
        return (torch.randn(*shape, generator=gen, device="cuda") * size).to(dtype)

    if layout == "fused":
        x = new(b, n, h + 2 * hk, d)
        return x[:, :, :h], x[:, :, h:h + hk], x[:, :, h + hk:], new(b, n, h, d)
    if layout == "heads_first":
        return tuple(new(b, hh, nn, d).transpose(1, 2) for hh, nn in ((h, n), (hk, m), (hk, m), (h, n)))
    if layout == "padded":                                   # rows longer than the heads, batch as the inner dimension
        return tuple(new(nn, b, hh, d + 8).transpose(0, 1)[..., :d] for hh, nn in ((h, n), (hk, m), (hk, m), (h, n)))
    return new(b, n, h, d), new(b, m, hk, d), new(b, m, hk, d), new(b, n, h, d)


CASES = [
    # b, n, m, h, hk, d, causal, dtype, layout
    (1, 128, 128, 1, 1, 64, False, torch.bfloat16, "plain"),
    (1, 128, 128, 1, 1, 128, False, torch.bfloat16, "plain"),
    (1, 1, 1, 1, 1, 64, False, torch.bfloat16, "plain"),
    (2, 1, 300, 4, 2, 128, True, torch.bfloat16, "plain"),
    (3, 77, 77, 4, 4, 64, False, torch.float16, "plain"),
    (2, 257, 257, 6, 2, 64, True, torch.float16, "fused"),
    (2, 129, 511, 4, 1, 96, True, torch.bfloat16, "heads_first"),
    (1, 511, 129, 4, 4, 72, True, torch.bfloat16, "padded"),      # most rows see nothing
    (2, 300, 40, 2, 1, 128, True, torch.float16, "plain"),        # a whole row tile sees nothing
    (2, 700, 700, 3, 1, 128, True, torch.bfloat16, "fused"),
    (1, 1000, 640, 2, 2, 128, False, torch.float16, "heads_first"),
    (1, 255, 383, 2, 1, 8, False, torch.bfloat16, "plain"),
    (1, 140, 140, 2, 2, 32, True, torch.float16, "plain"),
    (1, 384, 2100, 8, 2, 64, True, torch.bfloat16, "padded"),
    (1, 2100, 256, 2, 1, 80, False, torch.bfloat16, "plain"),
    (5, 64, 64, 2, 1, 120, True, torch.bfloat16, "plain"),
    (1, 1, 5000, 4, 2, 128, True, torch.bfloat16, "plain"),       # few rows, many keys: CTAs share them
    (2, 3, 2049, 2, 1, 64, False, torch.float16, "heads_first"),
    (1, 130, 3333, 1, 1, 96, True, torch.bfloat16, "plain"),
    (1, 1500, 1500, 2, 1, 128, True, torch.float16, "fused"),
    (1, 3000, 70, 3, 3, 64, False, torch.bfloat16, "plain"),
]


@pytest.mark.gpu
@pytest.mark.parametrize("case", CASES, ids=lambda c: "x".join(map(str, c[:6])) + f"_{'causal' if c[6] else 'full'}_{str(c[7])[6:]}_{c[8]}")
def test_matches_the_formulas(case):
    b, n, m, h, hk, d, causal, dtype, layout = case
    q, k, v, g = make(b, n, m, h, hk, d, dtype, layout)
    out, lse = fb.fewbit_attention_fwd(q, k, v, causal=causal)
    dq, dk, dv = fb.fewbit_attention_bwd(g, q, k, v, out, lse, causal=causal)
    assert fb.fewbit_attention_timeout_count() == 0
    for i in range(b):
        compare(q[i], k[i], v[i], g[i], {"out": out[i], "lse": lse[i], "dq": dq[i], "dk": dk[i], "dv": dv[i]}, causal, d ** -0.5)


@pytest.mark.gpu
def test_large_scores_move_the_reference_of_the_sums():
    """Scores that grow along the keys: the running maximum passes its reference again and again."""
    q, k, v, g = make(1, 200, 1500, 2, 1, 64, torch.bfloat16, seed=3)
    k = k * torch.linspace(0.05, 6, 1500, device="cuda")[None, :, None, None].bfloat16()
    out, lse = fb.fewbit_attention_fwd(q, k, v, scale=0.5)
    dq, dk, dv = fb.fewbit_attention_bwd(g, q, k, v, out, lse, scale=0.5)
    compare(q[0], k[0], v[0], g[0], {"out": out[0], "lse": lse[0]}, False, 0.5)
    assert all(x.isfinite().all() for x in (dq, dk, dv))


@pytest.mark.gpu
@pytest.mark.parametrize("dtype,d,h,hk", [(torch.bfloat16, 128, 4, 2), (torch.float16, 64, 3, 3)])
@pytest.mark.parametrize("causal", [False, True])
def test_packed_sequences(dtype, d, h, hk, causal):
    """Sequences of unequal lengths side by side, empty ones among them; rows of no sequence in front, between and behind,
    filled with NaN; query and key lengths that differ."""
    lens = [(1, 1), (130, 130), (0, 0), (257, 300), (5, 0), (0, 40), (64, 200), (300, 20)]
    qo, ko = [3], [7]
    for a, c in lens:
        qo.append(qo[-1] + a), ko.append(ko[-1] + c)
    q, k, v, g = (x[0].clone() for x in make(1, qo[-1] + 50, ko[-1] + 9, h, hk, d, dtype, seed=5))
    for x, lo, hi in ((q, 3, qo[-1]), (g, 3, qo[-1]), (k, 7, ko[-1]), (v, 7, ko[-1])):
        x[:lo] = float("nan")
        x[hi:] = float("nan")
    kw = dict(causal=causal, q_offsets=torch.tensor(qo, dtype=torch.int32, device="cuda"),
              k_offsets=torch.tensor(ko, dtype=torch.int32, device="cuda"), max_q_len=300, max_k_len=300)
    out, lse = fb.fewbit_attention_fwd(q, k, v, **kw)
    dq, dk, dv = fb.fewbit_attention_bwd(g, q, k, v, out, lse, **kw)
    assert fb.fewbit_attention_timeout_count() == 0
    for i in range(len(lens)):
        a, c = slice(qo[i], qo[i + 1]), slice(ko[i], ko[i + 1])
        compare(q[a], k[c], v[c], g[a], {"out": out[a], "lse": lse[:, a], "dq": dq[a], "dk": dk[c], "dv": dv[c]}, causal, d ** -0.5)
    for x in (out, dq):
        assert (x[:3] == 0).all() and (x[qo[-1]:] == 0).all()
    for x in (dk, dv):
        assert (x[:7] == 0).all() and (x[ko[-1]:] == 0).all()


@pytest.mark.gpu
def test_neighbouring_sequences_that_are_not_finite_do_not_leak():
    """The tile behind a sequence's end holds its neighbour's infinities and NaN."""
    lens = [100, 140, 70]
    o = [0, 100, 240, 310]
    q, k, v, g = (x[0].clone() for x in make(1, 310, 310, 2, 1, 64, torch.bfloat16, seed=6))
    for x in (q, k, v, g):
        x[100:240, :, ::3] = float("nan")
        x[100:240, :, 1::3] = float("inf")
    off = torch.tensor(o, dtype=torch.int32, device="cuda")
    kw = dict(causal=False, q_offsets=off, k_offsets=off, max_q_len=140, max_k_len=140)
    out, lse = fb.fewbit_attention_fwd(q, k, v, **kw)
    dq, dk, dv = fb.fewbit_attention_bwd(g, q, k, v, out, lse, **kw)
    for i in (0, 2):
        a = slice(o[i], o[i + 1])
        compare(q[a], k[a], v[a], g[a], {"out": out[a], "lse": lse[:, a], "dq": dq[a], "dk": dk[a], "dv": dv[a]}, False, 64 ** -0.5)
    assert out[100:240].isnan().any()


@pytest.mark.gpu
def test_offsets_outside_the_tensors_are_cut():
    q, k, v, g = (x[0].clone() for x in make(1, 200, 200, 2, 1, 64, torch.bfloat16, seed=7))
    off = torch.tensor([-50, 120, 100000], dtype=torch.int32, device="cuda")
    kw = dict(q_offsets=off, k_offsets=off, max_q_len=200, max_k_len=200)
    out, lse = fb.fewbit_attention_fwd(q, k, v, **kw)
    dq, dk, dv = fb.fewbit_attention_bwd(g, q, k, v, out, lse, **kw)
    for a in (slice(0, 120), slice(120, 200)):
        compare(q[a], k[a], v[a], g[a], {"out": out[a], "lse": lse[:, a], "dq": dq[a], "dk": dk[a], "dv": dv[a]}, False, 64 ** -0.5)


@pytest.mark.gpu
def test_other_stream_and_repeatability():
    q, k, v, g = make(2, 600, 600, 4, 2, 64, torch.bfloat16, seed=8)
    out, lse = fb.fewbit_attention_fwd(q, k, v, causal=True)
    one = (out, lse) + fb.fewbit_attention_bwd(g, q, k, v, out, lse, causal=True)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    out2, lse2 = fb.fewbit_attention_fwd(q, k, v, causal=True, stream=side)
    two = (out2, lse2) + fb.fewbit_attention_bwd(g, q, k, v, out2, lse2, causal=True, stream=side)
    torch.cuda.current_stream().wait_stream(side)
    assert all(torch.equal(a, b) for a, b in zip(one, two))


@pytest.mark.gpu
def test_gradients_against_differences():
    """Directional differences of the forward pass along 16-bit-representable steps.  The forward pass rounds P and out to
    2^-11 (binary16): with a step of 2^-3 on unit inputs, the second-order central difference is off by the third derivative
    (h^2 ~ 1.6e-2 of the value's scale) and by rounding: the loss sums 64 x 64 values whose errors 2^-11 |g out| are
    independent, 2^-11 x 64 / (2 h) = 0.13.  The bound is 0.3 + 5 %."""
    q, k, v, g = make(1, 64, 64, 1, 1, 64, torch.float16, seed=9)
    q, k = q / 2, k / 2
    out, lse = fb.fewbit_attention_fwd(q, k, v, causal=True)
    grads = fb.fewbit_attention_bwd(g, q, k, v, out, lse, causal=True)
    gen = torch.Generator(device="cuda").manual_seed(10)
    h = 2.0 ** -3
    for which in range(3):
        step = torch.sign(torch.randn(q.shape, generator=gen, device="cuda")).half() * (torch.rand(q.shape, generator=gen, device="cuda") < 0.05)
        ends = []
        for s in (h, -h):
            t = [q, k, v]
            t[which] = (t[which].float() + s * step).half()
            moved = t[which].double() - [q, k, v][which].double()
            ends.append(((fb.fewbit_attention_fwd(*t, causal=True)[0].double() * g.double()).sum(), moved))
        diff = float(ends[0][0] - ends[1][0])
        want = float((grads[which].double() * (ends[0][1] - ends[1][1])).sum())
        assert abs(diff - want) <= 0.3 * 2 * h + 0.05 * abs(want), which


@pytest.mark.gpu
def test_binding_refuses_what_does_not_match():
    q, k, v, g = make(1, 16, 16, 4, 2, 64, torch.bfloat16)
    with pytest.raises(ValueError):
        fb.fewbit_attention_fwd(q.float(), k.float(), v.float())
    with pytest.raises(ValueError):
        fb.fewbit_attention_fwd(q, k, v.half())
    with pytest.raises(ValueError):
        fb.fewbit_attention_fwd(q, k, v[:, :8])
    with pytest.raises(ValueError):
        fb.fewbit_attention_fwd(q, k, v, q_offsets=torch.zeros(2, dtype=torch.int32, device="cuda"))
    with pytest.raises(ValueError):
        fb.fewbit_attention_fwd(q.transpose(2, 3).contiguous().transpose(2, 3), k, v)
    with pytest.raises(fb.FewbitError) as e:
        fb.fewbit_attention_fwd(q[:, :, :3].contiguous(), k, v)
    assert e.value.status == 1
    with pytest.raises(fb.FewbitError) as e:
        fb.fewbit_attention_fwd(q[..., :12].contiguous(), k[..., :12].contiguous(), v[..., :12].contiguous())
    assert e.value.status == 2
    out, lse = fb.fewbit_attention_fwd(q, k, v)
    with pytest.raises(ValueError):
        fb.fewbit_attention_bwd(g, q, k, v, out, lse[:, :2])
    out, lse = fb.fewbit_attention_fwd(q[:, :0], k, v)
    assert out.numel() == 0 and lse.numel() == 0
    out, lse = fb.fewbit_attention_fwd(q, k[:, :0], v[:, :0])
    assert (out == 0).all() and (lse == -math.inf).all()


def test_library_refusals_need_no_gpu():
    lib = fb.load_library()
    A = 1 << 20
    H = ops._Heads

    def call(tensor=H(A, 1 << 16, 1024, 128), lse=A, ws=A, ws_bytes=1 << 20, **kw):
        base = dict(batch=2, heads=4, kv_heads=2, head_dim=128, q_len=100, k_len=100, causal=1, scale=0.1, dtype=1)
        s = ops._AttentionShape(**(base | kw))
        r = ctypes.byref(tensor)
        one = lib.fewbit_attention_fwd(ctypes.byref(s), r, r, r, r, lse, None)
        two = lib.fewbit_attention_bwd(ctypes.byref(s), r, r, r, r, r, lse, r, r, r, ws, ws_bytes, None)
        return one, two

    for kw in ({"batch": -1}, {"heads": 3}, {"kv_heads": 0}, {"q_len": -1}, {"scale": 0.0}, {"scale": float("nan")}, {"scale": float("inf")},
               {"dtype": 7}, {"head_dim": 0}, {"q_offsets": A}, {"q_offsets": A, "k_offsets": A, "q_rows": 50, "k_rows": 100}):
        assert call(**kw) == (1, 1), kw
    assert call(dtype=0) == (2, 2) and call(head_dim=136) == (2, 2) and call(head_dim=100) == (2, 2)
    assert call(q_len=1 << 31) == (6, 6) and call(heads=1 << 16, kv_heads=1 << 16, batch=1 << 16) == (6, 6)
    assert call(H(A + 8, 1 << 16, 1024, 128)) == (3, 3) and call(H(A, 1 << 16, 1023, 128)) == (3, 3)
    assert call(H(A, 1 << 16, 1024, -128)) == (2, 2) and call(H(A, 0, 1024, 128)) == (2, 2)
    assert call(H(None, 1 << 16, 1024, 128)) == (1, 1) and call(lse=None) == (1, 1) and call(lse=A + 2) == (3, 3)
    assert call(q_offsets=A + 2, k_offsets=A, q_rows=200, k_rows=200) == (3, 3)
    assert call(heads=0) == (0, 0) and call(batch=0) == (0, 0)
    s = ops._AttentionShape(batch=2, heads=4, kv_heads=2, head_dim=128, q_len=100, k_len=100, scale=0.1, dtype=1)
    assert lib.fewbit_attention_workspace_bytes(ctypes.byref(s)) == 2 * 4 * 1024        # 1 KB for each row tile
    r = ctypes.byref(H(A, 1 << 16, 1024, 128))
    args = [ctypes.byref(s), r, r, r, r, r, A, r, r, r]
    assert lib.fewbit_attention_bwd(*args, None, 0, None) == 1
    assert lib.fewbit_attention_bwd(*args, A + 8, 1 << 20, None) == 3
    assert lib.fewbit_attention_bwd(*args, A, 100, None) == 5
