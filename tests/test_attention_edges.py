"""Attention where it meets an edge: rows of one key, memory that belongs to no sequence, gradients of scores far apart, values
that are not a number, no heads."""
import ctypes
import math

import pytest
import torch

import paper_2202_00441_b200 as fb
import test_attention as ta
from paper_2202_00441_b200 import operators as ops

pytestmark = pytest.mark.gpu
NAN = float("nan")


# ---- rows that see one key: P = 1 whatever the score, so dS, dQ and their share of dK are exactly zero ---------------------
ONE_KEY = [
    # b, n, m, h, hk, d, causal, dtype
    (1, 1, 1, 1, 1, 64, True, torch.bfloat16),
    (3, 1, 1, 8, 2, 128, False, torch.float16),
    (3, 2035, 1, 6, 2, 64, True, torch.bfloat16),                 # only the last row sees the key
    (2, 322, 1, 4, 1, 96, False, torch.bfloat16),
    (2, 257, 257, 4, 2, 128, True, torch.bfloat16),               # row 0 of a causal sequence
    (1, 300, 40, 2, 1, 64, True, torch.float16),                  # row 260
    (1, 2100, 2100, 2, 1, 128, True, torch.bfloat16),             # tiles shared by clusters
    (1, 1500, 1500, 6, 1, 72, True, torch.float16),
]


@pytest.mark.parametrize("case", ONE_KEY, ids=lambda c: "x".join(map(str, c[:6])) + f"_{'causal' if c[6] else 'full'}_{str(c[7])[6:]}")
def test_rows_of_one_key_have_no_score_gradient(case):
    b, n, m, h, hk, d, causal, dtype = case
    q, k, v, g = ta.make(b, n, m, h, hk, d, dtype, seed=11)
    q = q * 8                                                     # scores of tens: the recomputed P is off by the most
    alone = torch.full((n,), m == 1, device="cuda")
    if causal:
        alone = (torch.arange(n, device="cuda") + m - n + 1).clamp(max=m) == 1
    assert alone.any()
    out, lse = fb.fewbit_attention_fwd(q, k, v, causal=causal)
    dq, dk, dv = fb.fewbit_attention_bwd(g, q, k, v, out, lse, causal=causal)
    assert (dq[:, alone] == 0).all()
    if m == 1:
        assert (dk == 0).all()
    g = g * alone[:, None, None]                                  # only those rows: nothing reaches dK, and key 0 has dV
    dq, dk, dv = fb.fewbit_attention_bwd(g, q, k, v, out, lse, causal=causal)
    assert (dq == 0).all() and (dk == 0).all()
    want = g.double().sum(1).view(b, hk, h // hk, d).sum(2)
    size = g.double().abs().sum(1).view(b, hk, h // hk, d).sum(2)
    assert ((dv[:, 0].double() - want).abs() <= 1.05 * ta.E[dtype] * (want.abs() + 2.0 ** -7 * size) + ta.TINY[dtype]).all()
    assert (dv[:, 1:] == 0).all()


def test_packed_sequences_of_one_token_have_no_score_gradient():
    n = 70
    q, k, v, g = (x[0] for x in ta.make(1, n, n, 4, 2, 64, torch.bfloat16, seed=12))
    off = torch.arange(n + 1, dtype=torch.int32, device="cuda")
    kw = dict(q_offsets=off, k_offsets=off, max_q_len=1, max_k_len=1)
    for causal in (False, True):
        out, lse = fb.fewbit_attention_fwd(q, k, v, causal=causal, **kw)
        dq, dk, dv = fb.fewbit_attention_bwd(g, q, k, v, out, lse, causal=causal, **kw)
        assert (dq == 0).all() and (dk == 0).all()
        assert torch.equal(out, v.repeat_interleave(2, 1))


def test_a_gradient_that_is_not_finite_shows_in_rows_of_one_key():
    q, k, v, g = ta.make(1, 4, 1, 2, 2, 64, torch.bfloat16, seed=13)
    g[0, 2, 1, 5] = NAN
    out, lse = fb.fewbit_attention_fwd(q, k, v)
    dq, dk, dv = fb.fewbit_attention_bwd(g, q, k, v, out, lse)
    assert dq[0, 2, 1].isnan().all() and dk[0, 0, 1].isnan().all() and dv[0, 0, 1, 5].isnan()
    assert (dq[0, :, 0] == 0).all() and (dk[0, 0, 0] == 0).all()


# ---- every row of a packed tensor is written --------------------------------------------------------------------------------
def _h(t):
    return ctypes.byref(ops._Heads(t.data_ptr(), 0, t.stride(0), t.stride(1)))


def packed_call(q_offsets, k_offsets, max_q, max_k, rows=150, keys=90, h=4, hk=2, d=64, causal=False):
    """Forward and backward pass through the C ABI into buffers full of NaN."""
    lib = fb.load_library()
    q, k, v, g = ta.make(1, rows, keys, h, hk, d, torch.bfloat16, seed=14)
    q, k, v, g = q[0], k[0], v[0], g[0]
    qo, ko = (torch.tensor(o, dtype=torch.int32, device="cuda") for o in (q_offsets, k_offsets))
    out, dq, dk, dv = (torch.full_like(t, NAN) for t in (q, q, k, v))
    lse = torch.full((h, rows), NAN, device="cuda")
    s = ops._AttentionShape(batch=len(q_offsets) - 1, heads=h, kv_heads=hk, head_dim=d, q_len=max_q, k_len=max_k, q_rows=rows, k_rows=keys,
                            q_offsets=qo.data_ptr(), k_offsets=ko.data_ptr(), causal=causal, scale=d ** -0.5, dtype=1)
    stream = torch.cuda.current_stream().cuda_stream
    assert lib.fewbit_attention_fwd(ctypes.byref(s), _h(q), _h(k), _h(v), _h(out), lse.data_ptr(), stream) == 0
    bytes_ = lib.fewbit_attention_workspace_bytes(ctypes.byref(s))
    ws = torch.full((bytes_ // 4 + 4,), NAN, device="cuda")
    assert lib.fewbit_attention_bwd(ctypes.byref(s), _h(g), _h(q), _h(k), _h(v), _h(out), lse.data_ptr(), _h(dq), _h(dk), _h(dv), ws.data_ptr(),
                                    bytes_, stream) == 0
    torch.cuda.synchronize()
    return (q, k, v, g), dict(out=out, lse=lse, dq=dq, dk=dk, dv=dv)


@pytest.mark.parametrize("offsets", [([0], [0]), ([40], [17]), ([5, 5, 5], [0, 0, 0]), ([0, 0], [90, 90])], ids=str)
@pytest.mark.parametrize("lens", [(0, 0), (150, 90), (0, 90), (150, 0)], ids=str)
def test_tensors_without_a_sequence_are_zeroed(offsets, lens):
    _, r = packed_call(*offsets, *lens)
    assert (r["lse"] == -math.inf).all()
    for name in ("out", "dq", "dk", "dv"):
        assert (r[name] == 0).all(), name


@pytest.mark.parametrize("lens", [(0, 90), (150, 0), (0, 0)], ids=str)
def test_a_bound_of_zero_on_one_side_leaves_nothing_unwritten(lens):
    """Sequences on the other side only: rows that see no key, keys that no row sees."""
    q_offsets = [0, 0, 0] if lens[0] == 0 else [10, 100, 150]
    k_offsets = [0, 0, 0] if lens[1] == 0 else [3, 50, 90]
    _, r = packed_call(q_offsets, k_offsets, *lens)
    assert (r["lse"] == -math.inf).all()
    for name in ("out", "dq", "dk", "dv"):
        assert (r[name] == 0).all(), name


@pytest.mark.parametrize("causal", [False, True])
def test_rows_past_the_length_bounds_are_zeroed(causal):
    """Sequences longer than max_q_len or max_k_len end there; what lies behind belongs to no sequence."""
    qo, ko, most_q, most_k = [2, 202, 262, 400], [1, 141, 146, 390], 128, 100
    x, r = packed_call(qo, ko, most_q, most_k, rows=420, keys=400, causal=causal)
    q, k, v, g = x
    inside_q, inside_k = torch.zeros(420, dtype=torch.bool, device="cuda"), torch.zeros(400, dtype=torch.bool, device="cuda")
    for i in range(3):
        a = slice(qo[i], min(qo[i + 1], qo[i] + most_q))
        c = slice(ko[i], min(ko[i + 1], ko[i] + most_k))
        inside_q[a], inside_k[c] = True, True
        ta.compare(q[a], k[c], v[c], g[a], {"out": r["out"][a], "lse": r["lse"][:, a], "dq": r["dq"][a], "dk": r["dk"][c], "dv": r["dv"][c]}, causal, 0.125)
    assert (r["lse"][:, ~inside_q] == -math.inf).all()
    for name, inside in (("out", inside_q), ("dq", inside_q), ("dk", inside_k), ("dv", inside_k)):
        assert (r[name][~inside] == 0).all(), name


def test_without_query_heads_the_key_gradients_are_zero():
    kv = torch.randn(2, 300, 2, 64, device="cuda").bfloat16()
    q = kv.new_empty(2, 300, 0, 64)
    out, lse = fb.fewbit_attention_fwd(q, kv, kv)
    full = [torch.full_like(kv, NAN) for _ in range(4)]           # what an allocation of that size finds
    del full
    dq, dk, dv = fb.fewbit_attention_bwd(q, q, kv, kv, out, lse)
    assert dq.shape == q.shape and (dk == 0).all() and (dv == 0).all()


# ---- values -----------------------------------------------------------------------------------------------------------------
@pytest.mark.parametrize("d", [64, 128])
def test_one_key_that_is_not_a_number_makes_the_rows_that_see_it_nan(d):
    """A softmax with one NaN is NaN throughout, its sum's logarithm too; rows that do not see the key keep their values.  Key i
    of head i is NaN, in two of three key tiles."""
    h, n = 128, 384
    q, k, v, _ = ta.make(1, n, n, h, h, d, torch.bfloat16, seed=15)
    clean = fb.fewbit_attention_fwd(q, k, v, causal=True)
    for first in (0, 128):
        bad = k.clone()
        at = torch.arange(h, device="cuda")
        bad[0, first + at, at] = NAN
        seen = torch.arange(n, device="cuda")[None] >= first + at[:, None]           # (head, row)
        for causal in (True, False):
            out, lse = fb.fewbit_attention_fwd(q, bad, v, causal=causal)
            sees = seen if causal else torch.ones_like(seen)
            assert lse[0][sees].isnan().all()
            assert out[0].transpose(0, 1)[sees].isnan().all()
            if causal:
                assert torch.equal(lse[0][~seen], clean[1][0][~seen])
                assert torch.equal(out[0].transpose(0, 1)[~seen], clean[0][0].transpose(0, 1)[~seen])


def test_gradients_of_scores_that_are_far_apart():
    """Scores of up to a hundred: P is nearly 0 or 1, and dS a difference of near values.  The bound of `compare` has delta's error
    (from the rounded output) in it; the scores' own rounding, 144 x 2^-24 in the exponent, is 2^-17 of P and below its 5 %."""
    q, k, v, g = ta.make(1, 200, 1500, 2, 1, 64, torch.bfloat16, seed=3)
    k = k * torch.linspace(0.05, 6, 1500, device="cuda")[None, :, None, None].bfloat16()
    out, lse = fb.fewbit_attention_fwd(q, k, v, scale=0.5)
    dq, dk, dv = fb.fewbit_attention_bwd(g, q, k, v, out, lse, scale=0.5)
    ta.compare(q[0], k[0], v[0], g[0], {"out": out[0], "lse": lse[0], "dq": dq[0], "dk": dk[0], "dv": dv[0]}, False, 0.5)


# ---- the count of waits that gave up ----------------------------------------------------------------------------------------
def test_the_timeout_count_waits_for_every_stream():
    x = torch.randn(8192, 8192, device="cuda").bfloat16()
    y = torch.empty_like(x)
    torch.mm(x, x, out=y)
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        for _ in range(200):                                      # some 140 ms
            torch.mm(x, x, out=y)
    assert fb.fewbit_attention_timeout_count() == 0
    assert side.query()
