"""Attention with shaped scores and the bias by buckets where they can go wrong beside ordinary values; tolerances as in
test_attention_scores.py."""
import math

import pytest
import torch

import paper_2202_00441_b200 as fb
import test_attention as ta
import test_attention_scores as ts

pytestmark = pytest.mark.gpu
BF, HALF = torch.bfloat16, torch.float16


@pytest.mark.parametrize("cap", [1e-30, 1e-50, 5e-324, 1e30, 1e39, 1e300, math.inf])
def test_caps_outside_the_range_are_refused(cap):
    """Those that binary32 rounds to 0 or infinity among them."""
    q, k, v, g = ta.make(1, 20, 20, 1, 1, 64, BF)
    with pytest.raises((fb.FewbitError, ValueError)):
        fb.fewbit_attention_fwd(q, k, v, cap=cap)
    with pytest.raises((fb.FewbitError, ValueError)):
        fb.fewbit_attention_bwd(g, q, k, v, q, torch.zeros(1, 1, 20, device="cuda"), cap=cap)


@pytest.mark.parametrize("b,n,m", [(2, 5, 0), (2, 0, 5), (2, 0, 0), (0, 5, 5)])
def test_documents_of_empty_sequences(b, n, m):
    i32 = {"dtype": torch.int32, "device": "cuda"}
    for mods in ({}, {"cap": 3.0, "distance_bias": torch.zeros(2, 7, device="cuda")}):
        q, k, v, g = ta.make(b, n, m, 2, 1, 64, BF)
        kw = {"q_documents": torch.zeros(b, n, **i32), "k_documents": torch.zeros(b, m, **i32), **mods}
        out, lse = fb.fewbit_attention_fwd(q, k, v, **kw)
        grads = fb.fewbit_attention_bwd(g, q, k, v, out, lse, **kw)
        assert (out == 0).all() and (lse == -math.inf).all() and all((x == 0).all() for x in grads)
    q, k, v, g = (x[0] for x in ta.make(1, n, m, 2, 1, 64, BF))
    kw = {"q_documents": torch.zeros(n, **i32), "k_documents": torch.zeros(m, **i32), "q_offsets": torch.tensor([0, n], **i32),
          "k_offsets": torch.tensor([0, m], **i32), "max_q_len": n, "max_k_len": m}
    if n and m:
        return
    out, lse = fb.fewbit_attention_fwd(q, k, v, **kw)
    grads = fb.fewbit_attention_bwd(g, q, k, v, out, lse, **kw)
    assert (out == 0).all() and (lse == -math.inf).all() and all((x == 0).all() for x in grads)


@pytest.mark.parametrize("both", [False, True])
@pytest.mark.parametrize("buckets,most", [(625, 3394), (624, 3394), (1024, 4095), (7, 8), (64, 2048), (512, 4096)])
def test_borders_of_buckets_that_almost_meet_a_distance(buckets, most, both):
    """625 buckets to 3394: (1524 / 312)^313 falls short of (3394 / 312)^208 by 2e-13 of it, so 1524 belongs below the border."""
    if both and buckets % 2:
        buckets *= 2
    if buckets > 1024:
        return
    table = torch.arange(buckets, device="cuda", dtype=torch.float32)[:, None]
    bias = fb.fewbit_relative_bias_fwd(table, most, bidirectional=both)
    assert torch.equal(bias[0].long(), ts.exact_buckets(buckets, most, both))


LARGE = [-1e3, -1e4, -1e6, -1e9, -1e30, -2e38, 1e6, 1e30]


@pytest.mark.parametrize("low", LARGE)
@pytest.mark.parametrize("case", [(1, 150, 150, 2, 2, 64, False, BF, {}), (2, 300, 280, 4, 2, 128, True, HALF, {}), (1, 130, 1500, 2, 1, 128, False, BF, {}),
                                  (1, 3, 2000, 4, 2, 64, True, HALF, {"prefix": 700}), (2, 200, 333, 2, 1, 96, False, HALF, {"docs": "sorted"}),
                                  (1, 3000, 70, 2, 1, 64, False, BF, {}), (1, 700, 700, 2, 1, 128, True, BF, {"docs": "scattered", "cap": 5.0}), (1, 1, 1, 1, 1, 8, True, BF, {})],
                         ids=lambda c: "x".join(map(str, c[:6])))
def test_rows_whose_biases_are_all_large(case, low):
    """Every key of the rows has the same large finite bias, and products are 0 (queries and keys in halves of the head that do not
    meet), so that the scores are equal whatever 32 bits leave of them: the results are those of a bias of 0.  (lse: one rounding to 32 bits
    of its own, and two of what it is computed from.)"""
    b, n, m, h, hk, d, causal, dtype, spec = case
    q, k, v, g = ta.make(b, n, m, h, hk, d, dtype)
    q[..., : d // 2] = 0
    k[..., d // 2:] = 0
    mods = ts.make_mods(b, n, m, h, spec)
    kw = {"causal": causal, **mods, "distance_bias": torch.full((h, 7), low, device="cuda")}
    out, lse = fb.fewbit_attention_fwd(q, k, v, **kw)
    grads = fb.fewbit_attention_bwd(g, q, k, v, out, lse, **kw)
    assert fb.fewbit_attention_timeout_count() == 0
    total = bound = 0
    for i in range(b):
        zero = {**ts.one(mods, i), "bias": torch.zeros(h, 7, device="cuda")}
        r, tol = ts.reference(*(x[i].double() for x in (q, k, v, g)), causal, d ** -0.5, **zero)
        fin = r["lse"] > -math.inf
        assert torch.equal(lse[i] > -math.inf, fin)
        want = r["lse"][fin] + low
        assert ((lse[i].double()[fin] - want).abs() <= 2.0 ** -22 * want.abs() + r["lse_tol"]).all()
        got = {"out": out[i], "dq": grads[0][i], "dk": grads[1][i], "dv": grads[2][i]}
        for name, x in got.items():
            limit = 1.05 * tol[name](ta.E[dtype], ta.TINY[dtype]).transpose(0, 1) + 1e-30
            err = (x.double() - r[name].transpose(0, 1)).abs()
            assert (err <= limit).all(), (name, float((err / limit).max()))
        total, bound = total + r["db"], bound + r["db_tol"]
    assert ((grads[3].double() - total).abs() <= bound + 1e-30).all()


@pytest.mark.parametrize("dtype", [BF, HALF], ids=str)
@pytest.mark.parametrize("docs", [None, "sorted"])
def test_rows_that_see_masked_keys_alone_beside_ordinary_ones(docs, dtype):
    """-1e9 beyond a distance of 40: the first rows, which lie further than that from every key, have nothing else, the others as if it were
    -inf.  A score of the first rows is what 32 bits leave of it, the bias alone: each of their keys has the same weight."""
    n, m, reach = 500, 250, 40
    q, k, v, g = ta.make(1, n, m, 2, 1, 64, dtype)
    kw = {} if docs is None else dict(zip(("q_documents", "k_documents"), ts.documents(docs, 1, n, m, 5)))
    bias = torch.randn(2, 2 * reach + 1, device="cuda")
    bias[:, 0] = bias[:, -1] = -1e9
    out, lse = fb.fewbit_attention_fwd(q, k, v, distance_bias=bias, **kw)
    grads = fb.fewbit_attention_bwd(g, q, k, v, out, lse, distance_bias=bias, **kw)
    # the same in two parts: rows with an ordinary key, by a table with -inf; the others, by products of 0
    away = torch.arange(m, device="cuda")[None] - torch.arange(n, device="cuda")[:, None] - (m - n)
    seen = torch.ones(n, m, dtype=torch.bool, device="cuda") if docs is None else kw["q_documents"][0][:, None] == kw["k_documents"][0][None]
    near = ((away.abs() < reach) & seen).any(1)
    assert near.any() and not near.all()
    hidden = bias.clone()
    hidden[:, 0] = hidden[:, -1] = -math.inf
    mods = {} if docs is None else {"qd": kw["q_documents"][0], "kd": kw["k_documents"][0]}
    args = [x[0].double() for x in (q, k, v, g)]
    ra, ta_ = ts.reference(*args, False, 0.125, bias=hidden, **mods)
    rb, tb_ = ts.reference(torch.zeros_like(args[0]), *args[1:], False, 0.125, bias=torch.zeros_like(bias), **mods)
    e, t = ta.E[dtype], ta.TINY[dtype]
    for name in ("out", "dq"):
        got = (out if name == "out" else grads[0])[0].double().transpose(0, 1)
        for r, tol, rows in ((ra, ta_, near), (rb, tb_, ~near)):
            assert ((got - r[name]).abs()[:, rows] <= (1.05 * tol[name](e, t) + 1e-30)[:, rows]).all(), name
    # dV, of which the second part's rows have P = 1 / n
    zero = args[3].clone()
    zero[~near] = 0
    parts = [ts.reference(args[0], args[1], args[2], zero, False, 0.125, bias=hidden, **mods)]
    zero = args[3].clone()
    zero[near] = 0
    parts.append(ts.reference(torch.zeros_like(args[0]), args[1], args[2], zero, False, 0.125, bias=torch.zeros_like(bias), **mods))
    want = sum(r["dv"] for r, _ in parts)
    limit = sum(tol["dv"](e, t) for _, tol in parts)
    assert ((grads[2][0].double().transpose(0, 1) - want).abs() <= 1.05 * limit + 1e-30).all()


@pytest.mark.parametrize("dtype", [BF, HALF], ids=str)
@pytest.mark.parametrize("table", [False, True])
@pytest.mark.parametrize("slope,first", [(1e38, 3), (3e38, 2)])
def test_slopes_whose_biases_overflow(slope, first, table, dtype):
    """Scores below what 32 bits hold, from distance `first` on, hide their keys: rows that lie further from every key see nothing, the
    others their nearest key alone (the next one's score is 1e38 lower), whose weight is 1 and whose score has no gradient."""
    n, m = 400, 128
    q, k, v, g = ta.make(1, n, m, 2, 1, 64, dtype)
    mods = {"slopes": torch.tensor([0.5, slope], device="cuda")}
    if table:
        mods["distance_bias"] = torch.zeros(2, 7, device="cuda")
    out, lse = fb.fewbit_attention_fwd(q, k, v, **mods)
    grads = fb.fewbit_attention_bwd(g, q, k, v, out, lse, **mods)
    assert all(torch.isfinite(x).all() for x in (out, *grads)) and torch.isfinite(lse[:, 0]).all()
    none = n - m - first + 1                                 # row i is n - m - i away from the first key
    assert (out[:, :none, 1] == 0).all() and (lse[:, 1, :none] == -math.inf).all() and (grads[0][:, :none, 1] == 0).all()
    nearest = torch.arange(none, n, device="cuda") - (n - m)
    assert torch.equal(out[:, none:, 1], v[:, nearest.clamp_min(0), 0]) and torch.isfinite(lse[:, 1, none:]).all()
    # dS is P (dP - delta), with delta off by the rounding of out at most
    size = (g[0, :, 1].double().abs() * out[0, :, 1].double().abs()).sum(-1, keepdim=True)
    assert (grads[0][0, :, 1].double().abs()[none:] <= 1.05 * 0.125 * (ta.E[dtype] * size[none:]) * k[0, nearest.clamp_min(0), 0].double().abs() + ta.TINY[dtype]).all()


@pytest.mark.parametrize("low", [-1e6, -1e9, 1e30])
@pytest.mark.parametrize("case", [([0, 40, 40, 300, 301], [0, 40, 50, 310, 310], 4, 2, 64, True, BF), ([5, 140, 300], [3, 140, 900], 4, 1, 128, False, HALF),
                                  ([0, 3, 5, 130, 258, 600], [0, 3, 4, 131, 259, 640], 2, 1, 96, True, HALF)], ids=lambda c: f"{len(c[0]) - 1}x{c[0][-1]}x{c[4]}")
def test_packed_rows_whose_biases_are_all_large_in_every_other_head(case, low):
    """As above; heads of one group take turns, and no row of another sequence is touched."""
    qo, ko, h, hk, d, causal, dtype = case
    b, extra = len(qo) - 1, 9
    q, k, v, g = (x[0] for x in ta.make(1, qo[-1] + extra, ko[-1] + extra, h, hk, d, dtype))
    q[..., : d // 2] = 0
    k[..., d // 2:] = 0
    bias = torch.zeros(h, 9, device="cuda")
    bias[1::2] = low
    offsets = [torch.tensor(o, dtype=torch.int32, device="cuda") for o in (qo, ko)]
    kw = {"causal": causal, "q_offsets": offsets[0], "k_offsets": offsets[1], "max_q_len": max(y - x for x, y in zip(qo, qo[1:])),
          "max_k_len": max(y - x for x, y in zip(ko, ko[1:])), "distance_bias": bias}
    out, lse = fb.fewbit_attention_fwd(q, k, v, **kw)
    grads = fb.fewbit_attention_bwd(g, q, k, v, out, lse, **kw)
    total = bound = 0
    for i in range(b):
        rows, keys = slice(qo[i], qo[i + 1]), slice(ko[i], ko[i + 1])
        r, tol = ts.reference(*(x.double() for x in (q[rows], k[keys], v[keys], g[rows])), causal, d ** -0.5, bias=torch.zeros_like(bias))
        for name, x in (("out", out[rows]), ("dq", grads[0][rows]), ("dk", grads[1][keys]), ("dv", grads[2][keys])):
            if x.numel():
                limit = 1.05 * tol[name](ta.E[dtype], ta.TINY[dtype]).transpose(0, 1) + 1e-30
                assert ((x.double() - r[name].transpose(0, 1)).abs() <= limit).all(), name
        total, bound = total + r["db"], bound + r["db_tol"]
    assert ((grads[3].double() - total).abs() <= bound + 1e-30).all()
    for x, at in ((out, qo), (grads[0], qo), (grads[1], ko), (grads[2], ko)):
        assert (x[:at[0]] == 0).all() and (x[at[-1]:] == 0).all()
    again = fb.fewbit_attention_bwd(g, q, k, v, out, lse, **kw)
    assert all(torch.equal(x, y) for x, y in zip(grads, again))


@pytest.mark.parametrize("low", [-1e4, -1e9, 1e30])
@pytest.mark.parametrize("case", [(1, 150, 150, 2, 2, 64, False, BF, {}), (2, 300, 280, 4, 2, 128, True, HALF, {}), (1, 3000, 70, 2, 1, 64, False, HALF, {}),
                                  (2, 200, 333, 2, 1, 96, False, HALF, {"docs": "sorted", "slopes": 0.0}), (1, 9, 900, 4, 1, 128, True, BF, {"cap": 5.0})],
                         ids=lambda c: "x".join(map(str, c[:6])))
def test_rows_whose_biases_are_all_large_without_the_biases_gradient(case, low):
    """The same, and dQ and dV bit for bit, where the workspace has no room for the rows' delta."""
    b, n, m, h, hk, d, causal, dtype, spec = case
    q, k, v, g = ta.make(b, n, m, h, hk, d, dtype)
    q[..., : d // 2] = 0
    k[..., d // 2:] = 0
    mods = ts.make_mods(b, n, m, h, spec)
    kw = {"causal": causal, **mods, "distance_bias": torch.full((h, 7), low, device="cuda")}
    out, lse = fb.fewbit_attention_fwd(q, k, v, **kw)
    dq, dk, dv = fb.fewbit_attention_bwd(g, q, k, v, out, lse, bias_grad=False, **kw)
    with_bias = fb.fewbit_attention_bwd(g, q, k, v, out, lse, **kw)
    assert torch.equal(dq, with_bias[0]) and torch.equal(dv, with_bias[2])
    for i in range(b):
        r, tol = ts.reference(*(x[i].double() for x in (q, k, v, g)), causal, d ** -0.5, **{**ts.one(mods, i), "bias": torch.zeros(h, 7, device="cuda")})
        limit = 1.05 * tol["dk"](ta.E[dtype], ta.TINY[dtype]).transpose(0, 1) + 1e-30
        assert ((dk[i].double() - r["dk"].transpose(0, 1)).abs() <= limit).all()


@pytest.mark.parametrize("dtype", [BF, HALF], ids=str)
@pytest.mark.parametrize("case", [(2, 1455, 3, 4, 1, 64, True, {"slopes": 3.0, "reach": 2000, "prefix": 2}), (1, 1700, 34, 4, 2, 8, False, {"slopes": 3.0, "reach": 1000, "cap": 3.0}),
                                  (1, 2200, 300, 2, 1, 128, False, {"slopes": 2.5, "reach": 60})], ids=lambda c: "x".join(map(str, c[:6])))
def test_gradients_of_biases_of_rows_far_from_every_key(case, dtype):
    """Slopes that bring lse past -2839, from where on a row's probabilities are found anew, and the rows' sums of dS with it in the bias's gradient: within the bound that z's own rounding leaves
    (2^-24 of its size, in units of ln 2), not delta's from rounded outputs."""
    b, n, m, h, hk, d, causal, spec = case
    q, k, v, g = ta.make(b, n, m, h, hk, d, dtype)
    mods = ts.make_mods(b, n, m, h, spec)
    kw = {"causal": causal, **mods}
    out, lse = fb.fewbit_attention_fwd(q, k, v, **kw)
    db = fb.fewbit_attention_bwd(g, q, k, v, out, lse, **kw)[3]
    total = bound = 0
    for i in range(b):
        r, _ = ts.reference(*(x[i].double() for x in (q, k, v, g)), causal, d ** -0.5, **ts.one(mods, i))
        size = float(r["lse"][r["lse"] > -math.inf].abs().max())
        # (db_tol's x, with a cap, leaves the size out; without one it is 2^5 of what this takes)
        x = 2.0 ** -18 * (1 + spec.get("cap", 0)) if "cap" in spec else 2.0 ** -19 * (1 + size)
        total, bound = total + r["db"], bound + r["db_tol"] * (2.0 ** -15 + 2.0 ** -18 * 4 + 2.0 ** -23 * size) / (2.0 ** -15 + x)
    assert float(lse[lse > -math.inf].min()) < -2839
    assert ((db.double() - total).abs() <= bound + 1e-30).all()
