"""Attention whose scores are capped, biased by distance and masked by prefix and documents, against the formulas in 64 bits; the
gradient of a bias by distance; the table by buckets; refusals.

Tolerances (derived).  As in test_attention.py: e = half a step of the 16-bit type, t its smallest step's half, P and dS rounded
once as operands, results once.  Further:
 z     is held in 32 bits in units of ln 2: off by 2^-22 of its size, the capped one by 2^-21 caps (the exponential unit's two
       results) more: P is off by x = 2^-19 (1 + max |z|) of itself, x = 2^-18 (1 + cap) with a cap.
 1 - t^2  is rounded to 11 bits (2^-12, or 2^-25 where it is small) and off by 2 t's error, 2^-20.
 dB    sums of P (dP - delta) in 32 bits: P off by 2^-17 (the exponential's polynomial 2^-18.5, lse's own rounding) and x, dP by
       2^-17 of A = |dO| |v| (128 terms), delta (corrected by the row's own sum) by as much of sum P A."""
import ctypes
import math

import pytest
import torch

import paper_2202_00441_b200 as fb
import test_attention as ta
from paper_2202_00441_b200 import binding, operators as ops

E, TINY = ta.E, ta.TINY
BF, HALF = torch.bfloat16, torch.float16


def exact_buckets(buckets, most, both):
    """Of the distances -most .. most, in whole numbers: (far / half)^(n - half) against (most / half)^step."""
    n = buckets // 2 if both else buckets
    half = n // 2
    of, step = [], 0
    for far in range(most + 1):
        while far >= half and step < n - half - 1 and far ** (n - half) * half ** (step + 1) >= most ** (step + 1) * half ** (n - half):
            step += 1
        of.append(far if far < half else half + step)
    ahead = [x + n for x in of[1:]] if both else [of[0]] * most
    return torch.tensor(of[:0:-1] + [of[0]] + ahead, device="cuda")


def reference(q, k, v, g, causal, scale, cap=0.0, slopes=None, bias=None, prefix=0, qd=None, kd=None):
    """One sequence, 64 bits: values, and the magnitudes that the tolerances need."""
    n, h, d = q.shape
    m, hk = k.shape[:2]
    dev = q.device
    q, g = (x.transpose(0, 1) for x in (q, g))
    k, v = (x.transpose(0, 1).repeat_interleave(h // hk, 0) for x in (k, v))
    z = scale * q @ k.transpose(1, 2)
    bend = torch.ones_like(z)
    if cap:
        t = (z / cap).tanh()
        z, bend = cap * t, 1 - t * t
    away = torch.arange(m, device=dev)[None] - torch.arange(n, device=dev)[:, None] - (m - n)
    if slopes is not None:
        z = z - slopes.double()[:, None, None] * away.abs()
    if bias is not None:
        r = bias.shape[1] // 2
        z = z + bias.double()[:, away.clamp(-r, r) + r]
    seen = torch.ones(n, m, dtype=torch.bool, device=dev)
    if causal:
        seen &= (away <= 0) | (torch.arange(m, device=dev)[None] < prefix)
    if qd is not None:
        seen &= qd[:, None] == kd[None]
    size = torch.where(seen & (z > -math.inf), z.abs(), 0.0).amax() if z.numel() else 0.0
    z = z.masked_fill(~seen, -math.inf)
    lse = torch.logsumexp(z, -1) if m else torch.full((h, n), -math.inf, dtype=torch.float64, device=dev)
    p = torch.where(z == -math.inf, 0.0, (z - torch.where(lse == -math.inf, 0.0, lse)[..., None]).exp())
    out = p @ v
    dp = g @ v.transpose(1, 2)
    delta = (g * out).sum(-1, keepdim=True)
    dz = p * (dp - delta)
    ds = dz * bend

    def shared(x):
        return x.view(hk, h // hk, *x.shape[1:]).sum(1)

    r = {"out": out, "lse": lse, "dq": scale * ds @ k, "dk": shared(scale * ds.transpose(1, 2) @ q), "dv": shared(p.transpose(1, 2) @ g)}
    x = 2.0 ** -18 * (1 + cap) if cap else 2.0 ** -19 * (1 + float(size))
    live = (z > -math.inf).double()
    off_delta = (g.abs() * out.abs()).sum(-1, keepdim=True)
    mag = g.abs() @ v.abs().transpose(1, 2)

    def ds_err(e, t):
        of_dz = (e + x) * (dz.abs() + p * off_delta + p * (e + x) * mag) + x * p * (dp.abs() + delta.abs()) + (t + p * t * g.abs().sum(-1, keepdim=True)) * live
        return of_dz * bend + dz.abs() * (2.0 ** -11 * bend + 2.0 ** -19) * (1 if cap else 0)

    tol = {
        "out": lambda e, t: ((e + x) * p + t * live) @ v.abs() + (e + x) * out.abs() + t,
        "dv": lambda e, t: shared(((e + x) * p + t * live).transpose(1, 2) @ g.abs()) + e * r["dv"].abs() + t,
        "dq": lambda e, t: scale * ds_err(e, t) @ k.abs() + e * r["dq"].abs() + t,
        "dk": lambda e, t: shared(scale * ds_err(e, t).transpose(1, 2) @ q.abs()) + e * r["dk"].abs() + t,
    }
    if bias is not None:
        reach = bias.shape[1] // 2
        at = (away.clamp(-reach, reach) + reach).flatten().expand(h, -1)
        zero = torch.zeros(h, 2 * reach + 1, dtype=torch.float64, device=dev)
        r["db"] = zero.scatter_add(1, at, dz.flatten(1))
        r["db_tol"] = (2.0 ** -15 + x) * zero.scatter_add(1, at, (p * (mag + (p * mag).sum(-1, keepdim=True))).flatten(1))
    r["lse_tol"] = 2.0 ** -16 + 2 * x
    return r, tol


def compare(q, k, v, g, got, causal, scale, **mods):
    dtype = q.dtype
    r, tol = reference(*(x.double() for x in (q, k, v, g)), causal, scale, **mods)
    assert torch.equal(got["lse"].double() == -math.inf, r["lse"] == -math.inf)
    fin = r["lse"] > -math.inf
    assert ((got["lse"].double() - r["lse"])[fin].abs() <= r["lse_tol"] * (1 + r["lse"][fin].abs())).all()
    for name in ("out", "dq", "dk", "dv"):
        if got[name].numel():
            bound = 1.05 * tol[name](E[dtype], TINY[dtype]).transpose(0, 1) + 1e-30
            err = (got[name].double() - r[name].transpose(0, 1)).abs()
            assert (err <= bound).all(), (name, float((err / bound).max()), float(err.max()))
    return r


def documents(kind, b, n, m, seed):
    gen = torch.Generator().manual_seed(seed)
    if kind == "sorted":                                     # a handful of documents, in order
        cut = lambda length: torch.randint(0, 5, (b, length), generator=gen).sort(1).values  # noqa: E731
        qd = cut(n)
        kd = qd.clone() if n == m else cut(m)
    elif kind == "alone":                                    # every row has a document of its own
        qd, kd = torch.arange(n).repeat(b, 1), torch.arange(m).repeat(b, 1)
    elif kind == "scattered":                                # any numbers in any order, negative ones and the largest too
        names = torch.tensor([-(1 << 31), -7, 0, 3, (1 << 31) - 1])
        qd, kd = names[torch.randint(0, 5, (b, n), generator=gen)], names[torch.randint(0, 5, (b, m), generator=gen)]
    elif kind == "strangers":                                # no row has a key
        qd, kd = torch.zeros(b, n), torch.ones(b, m)
    elif kind == "falling":                                  # runs of many different numbers, falling
        qd, kd = -(torch.arange(n) // 37).repeat(b, 1), -(torch.arange(m) // 37).repeat(b, 1)
    elif kind == "late":                                     # the keys that count come last
        qd, kd = torch.zeros(b, n), (torch.arange(m) < m - 100).repeat(b, 1)
    return qd.int().cuda(), kd.int().cuda()


def make_mods(b, n, m, h, spec, seed=3):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    mods = {}
    if "cap" in spec:
        mods["cap"] = spec["cap"]
    if "slopes" in spec:
        mods["slopes"] = torch.rand(h, generator=gen, device="cuda") * spec["slopes"]
    if "reach" in spec:
        mods["distance_bias"] = torch.randn(h, 2 * spec["reach"] + 1, generator=gen, device="cuda")
        if spec.get("hide"):                                 # some distances hidden, the far ones of a head among them
            mods["distance_bias"][:, ::5] = -math.inf
            mods["distance_bias"][0, 0] = mods["distance_bias"][0, -1] = -math.inf
    if "prefix" in spec:
        mods["prefix_lens"] = torch.tensor([spec["prefix"] // (i + 1) for i in range(b)], dtype=torch.int32, device="cuda")
    if "docs" in spec:
        mods["q_documents"], mods["k_documents"] = documents(spec["docs"], b, n, m, seed)
    return mods


def one(mods, i):
    """Of sequence i of a batch, as the reference takes it."""
    r = {"cap": mods.get("cap", 0.0), "slopes": mods.get("slopes"), "bias": mods.get("distance_bias")}
    if "prefix_lens" in mods:
        r["prefix"] = int(mods["prefix_lens"][i])
    if "q_documents" in mods:
        r["qd"], r["kd"] = mods["q_documents"][i], mods["k_documents"][i]
    return r


def check_all(b, n, m, h, hk, d, causal, dtype, layout, mods, scale=None, size=1.0):
    q, k, v, g = ta.make(b, n, m, h, hk, d, dtype, layout, size=size)
    kw = {"causal": causal, "scale": scale, **mods}
    out, lse = fb.fewbit_attention_fwd(q, k, v, **kw)
    grads = fb.fewbit_attention_bwd(g, q, k, v, out, lse, **kw)
    assert fb.fewbit_attention_timeout_count() == 0
    total = bound = 0
    for i in range(b):
        got = {"out": out[i], "lse": lse[i], "dq": grads[0][i], "dk": grads[1][i], "dv": grads[2][i]}
        r = compare(q[i], k[i], v[i], g[i], got, causal, scale or d ** -0.5, **one(mods, i))
        if "db" in r:
            total, bound = total + r["db"], bound + r["db_tol"]
    if "distance_bias" in mods:
        assert len(grads) == 4 and grads[3].dtype == torch.float32
        err = (grads[3].double() - total).abs()
        assert (err <= bound + 1e-30).all(), (float((err / (bound + 1e-30)).max()), float(err.max()))
        same = fb.fewbit_attention_bwd(g, q, k, v, out, lse, bias_grad=False, **kw)
        assert len(same) == 3 and torch.equal(same[0], grads[0]) and torch.equal(same[2], grads[2])
    else:
        assert len(grads) == 3
    again = fb.fewbit_attention_bwd(g, q, k, v, out, lse, **kw)
    assert all(torch.equal(x, y) for x, y in zip(grads, again))


CASES = [
    # b, n, m, h, hk, d, causal, dtype, layout, what
    (1, 128, 128, 1, 1, 64, False, BF, "plain", {"cap": 30.0}),
    (1, 1, 1, 1, 1, 64, True, BF, "plain", {"cap": 5.0, "slopes": 1.0, "reach": 3, "prefix": 1}),
    (2, 77, 77, 4, 4, 64, True, HALF, "plain", {"cap": 30.0}),
    (1, 300, 300, 2, 1, 128, True, BF, "fused", {"cap": 0.5}),                       # every score far past the cap
    (2, 257, 300, 2, 2, 96, False, HALF, "heads_first", {"cap": 4.0}),
    (2, 200, 333, 6, 2, 64, True, BF, "plain", {"slopes": 0.5}),
    (1, 333, 200, 3, 1, 128, False, HALF, "padded", {"slopes": 0.1}),
    (1, 513, 513, 2, 1, 64, True, BF, "plain", {"prefix": 200}),
    (3, 140, 400, 2, 2, 32, True, HALF, "plain", {"prefix": 399}),
    (2, 400, 130, 2, 1, 128, True, BF, "plain", {"prefix": 1}),                      # most rows see key 0 alone
    (2, 300, 300, 4, 2, 64, True, BF, "plain", {"docs": "sorted"}),
    (1, 700, 500, 2, 1, 128, False, HALF, "plain", {"docs": "sorted"}),
    (1, 300, 300, 2, 1, 128, True, BF, "plain", {"docs": "alone"}),
    (2, 200, 450, 2, 2, 72, False, BF, "plain", {"docs": "scattered"}),
    (1, 200, 450, 2, 1, 64, True, HALF, "plain", {"docs": "strangers"}),
    (1, 900, 900, 1, 1, 128, True, BF, "plain", {"docs": "falling"}),
    (1, 130, 1500, 2, 1, 128, False, BF, "plain", {"docs": "late"}),                 # one row tile, CTAs share the keys
    (1, 1, 5000, 2, 1, 64, True, HALF, "plain", {"docs": "late", "cap": 20.0}),
    (1, 3, 4000, 4, 2, 128, True, BF, "plain", {"cap": 20.0, "slopes": 0.01}),
    (2, 256, 256, 2, 2, 64, False, BF, "plain", {"reach": 128}),
    (1, 333, 517, 4, 4, 64, True, HALF, "plain", {"reach": 128}),
    (2, 517, 333, 4, 2, 128, False, BF, "plain", {"reach": 20}),
    (1, 600, 600, 2, 1, 64, True, BF, "plain", {"reach": 1}),
    (1, 260, 130, 2, 1, 128, False, HALF, "plain", {"reach": 4096}),
    (2, 100, 700, 3, 1, 64, False, BF, "plain", {"reach": 300}),
    (1, 3000, 70, 2, 1, 64, False, BF, "plain", {"reach": 60}),                      # one key tile, CTAs share the rows
    (1, 1000, 129, 4, 1, 128, True, BF, "plain", {"reach": 40}),
    (1, 300, 300, 2, 1, 64, False, BF, "plain", {"reach": 50, "hide": True}),
    (1, 400, 400, 2, 2, 128, True, HALF, "plain", {"reach": 100, "cap": 10.0}),
    (2, 300, 280, 4, 2, 64, True, BF, "plain", {"reach": 30, "cap": 3.0, "slopes": 0.02, "prefix": 100, "docs": "sorted"}),
    (2, 150, 150, 2, 1, 128, False, BF, "plain", {"reach": 200, "docs": "scattered"}),
    (1, 1, 300, 2, 1, 64, False, HALF, "plain", {"reach": 7, "docs": "late"}),
    (1, 1300, 1300, 2, 1, 8, True, BF, "plain", {"cap": 15.0, "docs": "sorted"}),
]


@pytest.mark.gpu
@pytest.mark.parametrize("case", CASES, ids=lambda c: "x".join(map(str, c[:6])) + f"_{'causal' if c[6] else 'full'}_{str(c[7])[6:]}_" + "_".join(f"{a}{x}" for a, x in c[9].items()))
def test_matches_the_formulas(case):
    b, n, m, h, hk, d, causal, dtype, layout, spec = case
    check_all(b, n, m, h, hk, d, causal, dtype, layout, make_mods(b, n, m, h, spec))


@pytest.mark.gpu
@pytest.mark.parametrize("cap", [2.0 ** -60, 2.0 ** -30, 2.0 ** 25, 2.0 ** 60])
def test_the_smallest_and_largest_caps(cap):
    """Every score next to 0, and scores as if there were no cap: nothing that is not finite comes out of squares and reciprocals."""
    q, k, v, g = ta.make(1, 150, 150, 2, 1, 64, BF)
    out, lse = fb.fewbit_attention_fwd(q, k, v, cap=cap)
    grads = fb.fewbit_attention_bwd(g, q, k, v, out, lse, cap=cap)
    assert all(torch.isfinite(x).all() for x in (out, lse, *grads))
    if cap < 1:
        assert ((lse.double() - math.log(150)).abs() <= 2.0 ** -18).all()
    else:
        plain = fb.fewbit_attention_fwd(q, k, v)
        assert ((lse - plain[1]).abs() <= 2.0 ** -16 * (1 + plain[1].abs())).all()


@pytest.mark.gpu
@pytest.mark.parametrize("cap,scale", [(200.0, 0.125), (300.0, 0.125), (5000.0, 1.0), (1e6, 0.01), (30.0, 0.001), (2e-4, 0.125)])
def test_caps_far_from_the_scale(cap, scale):
    """On both sides of where scale and cap fold into the polynomials' coefficients: the scores' relative error stays below 2^-19, so
    that lse is within 2^-18 (1 + largest score)."""
    q, k, _, _ = ta.make(1, 200, 200, 1, 1, 64, BF, size=2.0)
    _, lse = fb.fewbit_attention_fwd(q, k, k, cap=cap, scale=scale)
    z = cap * (scale * q[0, :, 0].double() @ k[0, :, 0].double().T / cap).tanh()
    assert ((lse[0, 0].double() - torch.logsumexp(z, 1)).abs() <= 2.0 ** -18 * (1 + z.abs().amax())).all()


@pytest.mark.gpu
@pytest.mark.parametrize("cap", [0.25, 2.0, 50.0])
def test_large_products_reach_the_cap(cap):
    """Products of a size of 100: both forms of the tanh, and slopes 1 - t^2 down to 0."""
    check_all(1, 200, 200, 2, 1, 64, True, BF, "plain", {"cap": cap}, size=3.0)
    check_all(1, 200, 200, 2, 1, 64, False, HALF, "plain", {"cap": cap}, scale=4.0)


@pytest.mark.gpu
@pytest.mark.parametrize("size", [1.0, 2.0])
def test_a_cap_costs_no_further_rounding_in_binary16(size):
    """dK has two roundings to 16 bits, dS's and its own, whose errors do not depend on one another: sqrt(2) times as far off, in the
    root mean square, as its own alone.  1 - t^2 in steps of 2^-15 (rms 2^-16 / sqrt(3) of at least 0.4) or with 13 bits (rms below
    2^-14 / sqrt(3)) brings that to at most 1.43, as binary16 (11 bits, near 1 an rms of 2^-12 / sqrt(3)) to 1.57 or more.  size 2:
    scores past the cap."""
    q, k, v, g = ta.make(2, 512, 512, 4, 4, 64, HALF, size=size)
    out, lse = fb.fewbit_attention_fwd(q, k, v, cap=5.0)
    _, dk, _ = fb.fewbit_attention_bwd(g, q, k, v, out, lse, cap=5.0)
    error = alone = 0.0
    for b in range(2):
        exact = reference(*(x[b].double() for x in (q, k, v, g)), False, 0.125, cap=5.0)[0]["dk"].transpose(0, 1)
        error += float((dk[b].double() - exact).square().sum())
        alone += float((exact.to(HALF).double() - exact).square().sum())
    assert error <= 1.5 ** 2 * alone, math.sqrt(error / alone)


@pytest.mark.gpu
@pytest.mark.parametrize("slopes", [False, True])
@pytest.mark.parametrize("size", [-1.4, 0.4, 1.4])
def test_one_large_product_at_every_place(size, slopes):
    """Sequence b has one product of `size` caps, at key b of row 5 + b, and zeros else: whichever form of the tanh it needs, the form
    that its neighbours would do with is not taken.  lse within 2^-18 (of sums of 130 terms: 2^-24 of 5, and the capped score's 2^-21)."""
    b, d, cap = 128, 128, 3.0
    q = torch.zeros(b, 140, 1, d, device="cuda", dtype=BF)
    k = torch.zeros(b, 130, 1, d, device="cuda", dtype=BF)
    at = torch.arange(b, device="cuda")
    k[:, :b, 0, :] = torch.eye(b, device="cuda", dtype=BF)
    q[at, 5 + at, 0, at] = size * cap
    mods = {"cap": cap, "scale": 1.0, **({"slopes": torch.zeros(1, device="cuda")} if slopes else {})}
    _, lse = fb.fewbit_attention_fwd(q, k, k, **mods)
    z = torch.zeros(b, 140, 130, dtype=torch.float64, device="cuda")
    z[at, 5 + at, at] = cap * (q[at, 5 + at, 0, at].double() / cap).tanh()
    assert ((lse[:, 0].double() - torch.logsumexp(z, 2)).abs() <= 2.0 ** -18).all()


PACKED = [
    ([0, 40, 40, 300, 301], [0, 40, 50, 310, 310], 4, 2, 64, True, BF, {"cap": 20.0}),
    ([0, 129, 400, 400, 1000], [0, 129, 400, 400, 1000], 2, 1, 128, True, BF, {"docs": "sorted", "cap": 10.0}),
    ([0, 129, 400, 777], [0, 300, 310, 900], 2, 2, 64, False, HALF, {"reach": 60}),
    ([0, 200, 200, 500], [0, 90, 95, 400], 4, 1, 96, True, BF, {"reach": 128, "slopes": 0.02, "prefix": 80, "docs": "scattered"}),
    ([5, 140, 300], [3, 140, 300], 2, 1, 64, True, BF, {"prefix": 300, "reach": 9}),   # rows in front of the first sequence
    ([0, 3, 5, 130, 258, 258, 600, 601], [0, 3, 4, 131, 259, 300, 640, 640], 4, 2, 64, False, BF, {"reach": 300}),   # tiles' places next to each other
    ([0, 512, 640, 650], [0, 384, 512, 1000], 2, 2, 128, False, HALF, {"reach": 40}),
]


@pytest.mark.gpu
@pytest.mark.parametrize("case", PACKED, ids=lambda c: f"{len(c[0]) - 1}x{c[0][-1]}x{c[4]}_" + "_".join(f"{a}{x}" for a, x in c[7].items()))
def test_packed_sequences(case):
    qo, ko, h, hk, d, causal, dtype, spec = case
    b, extra = len(qo) - 1, 11                               # rows behind the last sequence, which belong to none
    n, m = qo[-1] + extra, ko[-1] + extra
    q, k, v, g = (x[0] for x in ta.make(1, n, m, h, hk, d, dtype))
    mods = make_mods(1, n, m, h, spec)
    if "prefix" in spec:
        mods["prefix_lens"] = torch.tensor([spec["prefix"] // (i + 1) for i in range(b)], dtype=torch.int32, device="cuda")
    if "docs" in spec:
        mods["q_documents"], mods["k_documents"] = mods["q_documents"][0], mods["k_documents"][0]
    offsets = [torch.tensor(o, dtype=torch.int32, device="cuda") for o in (qo, ko)]
    kw = {"causal": causal, "q_offsets": offsets[0], "k_offsets": offsets[1], "max_q_len": max(y - x for x, y in zip(qo, qo[1:])),
          "max_k_len": max(y - x for x, y in zip(ko, ko[1:])), **mods}
    out, lse = fb.fewbit_attention_fwd(q, k, v, **kw)
    grads = fb.fewbit_attention_bwd(g, q, k, v, out, lse, **kw)
    total = bound = 0
    for i in range(b):
        rows, keys = slice(qo[i], qo[i + 1]), slice(ko[i], ko[i + 1])
        one_of = {"cap": mods.get("cap", 0.0), "slopes": mods.get("slopes"), "bias": mods.get("distance_bias")}
        if "prefix" in spec:
            one_of["prefix"] = int(mods["prefix_lens"][i])
        if "docs" in spec:
            one_of["qd"], one_of["kd"] = mods["q_documents"][rows], mods["k_documents"][keys]
        got = {"out": out[rows], "lse": lse[:, rows], "dq": grads[0][rows], "dk": grads[1][keys], "dv": grads[2][keys]}
        r = compare(q[rows], k[keys], v[keys], g[rows], got, causal, d ** -0.5, **one_of)
        if "db" in r:
            total, bound = total + r["db"], bound + r["db_tol"]
    for x, at in ((out, qo), (grads[0], qo), (grads[1], ko), (grads[2], ko)):
        assert (x[:at[0]] == 0).all() and (x[at[-1]:] == 0).all()
    if "reach" in spec:
        assert ((grads[3].double() - total).abs() <= bound + 1e-30).all()


@pytest.mark.gpu
def test_what_documents_hide_may_be_loud():
    """Keys of other documents whose scores would overflow the exponential, and queries past it: they change nothing."""
    q, k, v, g = ta.make(1, 256, 256, 2, 1, 64, BF)
    qd = (torch.arange(256, device="cuda") // 100)[None].int()
    loud = k.clone()
    loud[:, 100:200] *= 1000
    for mods in ({"q_documents": qd, "k_documents": qd}, {"q_documents": qd, "k_documents": qd, "distance_bias": torch.zeros(2, 11, device="cuda")}):
        a = fb.fewbit_attention_fwd(q, k, v, **mods)
        b = fb.fewbit_attention_fwd(q, loud, v, **mods)
        rows = torch.cat([torch.arange(100), torch.arange(200, 256)]).cuda()
        assert torch.equal(a[0][:, rows], b[0][:, rows]) and torch.equal(a[1][:, :, rows], b[1][:, :, rows])
        ga, gb = fb.fewbit_attention_bwd(g, q, k, v, *a, **mods), fb.fewbit_attention_bwd(g, q, loud, v, *b, **mods)
        assert all(torch.equal(x[:, rows], y[:, rows]) for x, y in zip(ga[:3], gb[:3])) and all(torch.isfinite(x).all() for x in gb)


@pytest.mark.gpu
def test_biases_that_hide_whole_rows():
    """-inf, or what 32 bits cannot hold in units of ln 2, at every distance: rows that see nothing."""
    q, k, v, g = ta.make(1, 150, 150, 2, 2, 64, BF)
    for low in (-math.inf, torch.finfo(torch.float32).min):
        bias = torch.zeros(2, 9, device="cuda")
        bias[1] = low
        out, lse = fb.fewbit_attention_fwd(q, k, v, distance_bias=bias)
        assert (out[:, :, 1] == 0).all() and (lse[:, 1] == -math.inf).all() and torch.isfinite(lse[:, 0]).all()
        grads = fb.fewbit_attention_bwd(g, q, k, v, out, lse, distance_bias=bias)
        assert all(torch.isfinite(x).all() for x in grads) and all((x[:, :, 1] == 0).all() for x in grads[:3]) and (grads[3][1] == 0).all()


@pytest.mark.gpu
def test_prefixes_out_of_range_are_cut():
    q, k, v, g = ta.make(2, 150, 200, 2, 1, 64, BF)
    for wild, tame in ((-5, 0), (1 << 30, 200), (-(1 << 31), 0)):
        a = fb.fewbit_attention_fwd(q, k, v, causal=True, prefix_lens=torch.tensor([wild, 77], dtype=torch.int32, device="cuda"))
        b = fb.fewbit_attention_fwd(q, k, v, causal=True, prefix_lens=torch.tensor([tame, 77], dtype=torch.int32, device="cuda"))
        assert torch.equal(a[0], b[0]) and torch.equal(a[1], b[1])


@pytest.mark.gpu
def test_scores_that_change_nothing_give_the_plain_results():
    """No cap (0 or None), slopes of 0, one document: within the plain scores' own roundings (another order of products)."""
    q, k, v, g = ta.make(2, 200, 260, 4, 2, 64, HALF)
    plain = fb.fewbit_attention_fwd(q, k, v, causal=True)
    for mods in ({"cap": 0.0}, {"cap": None}):
        got = fb.fewbit_attention_fwd(q, k, v, causal=True, **mods)
        assert torch.equal(got[0], plain[0]) and torch.equal(got[1], plain[1])
    check_all(2, 200, 260, 4, 2, 64, True, HALF, "plain", {"slopes": torch.zeros(4, device="cuda"), "prefix_lens": torch.zeros(2, dtype=torch.int32, device="cuda"),
                                                           "q_documents": torch.zeros(2, 200, dtype=torch.int32, device="cuda"),
                                                           "k_documents": torch.zeros(2, 260, dtype=torch.int32, device="cuda")})


@pytest.mark.gpu
def test_empty_sizes():
    for b, n, m, h in ((0, 5, 5, 2), (2, 0, 5, 2), (2, 5, 0, 2), (2, 0, 0, 2), (1, 5, 5, 0)):
        q, k, v, g = ta.make(b, n, m, h, 0 if h == 0 else 1, 64, BF)
        mods = {"distance_bias": torch.zeros(h, 7, device="cuda"), "cap": 3.0}
        out, lse = fb.fewbit_attention_fwd(q, k, v, **mods)
        grads = fb.fewbit_attention_bwd(g, q, k, v, out, lse, **mods)
        assert (grads[3] == 0).all() and grads[3].shape == (h, 7) and (grads[1] == 0).all()
        if m == 0:
            assert (out == 0).all() and (lse == -math.inf).all()
    q, k, v, g = (x[0] for x in ta.make(1, 9, 9, 2, 1, 64, BF))  # packed, of no sequence, and of empty ones
    for offsets in ([0], [0, 0, 0], [9, 9]):
        o = torch.tensor(offsets, dtype=torch.int32, device="cuda")
        mods = {"distance_bias": torch.zeros(2, 7, device="cuda"), "q_documents": torch.zeros(9, dtype=torch.int32, device="cuda"),
                "k_documents": torch.zeros(9, dtype=torch.int32, device="cuda"), "q_offsets": o, "k_offsets": o}
        for longest in (0, 9):
            kw = {**mods, "max_q_len": longest, "max_k_len": longest}
            out, lse = fb.fewbit_attention_fwd(q, k, v, **kw)
            grads = fb.fewbit_attention_bwd(g, q, k, v, out, lse, **kw)
            assert (out == 0).all() and all((x == 0).all() for x in grads)


@pytest.mark.gpu
def test_captured_graphs_and_other_streams():
    """Two graphs of calls that share no workspace, replayed in turn with new masks in the same buffers; a call on a side stream."""
    q, k, v, g = ta.make(2, 150, 200, 4, 2, 64, BF)
    table = torch.randn(32, 4, device="cuda")
    docs = [torch.zeros(2, n, dtype=torch.int32, device="cuda") for n in (150, 200)]

    def step(cap):
        bias = fb.fewbit_relative_bias_fwd(table, 60, bidirectional=True)
        mods = {"distance_bias": bias, "q_documents": docs[0], "k_documents": docs[1], "cap": cap}
        out, lse = fb.fewbit_attention_fwd(q, k, v, **mods)
        grads = fb.fewbit_attention_bwd(g, q, k, v, out, lse, **mods)
        return (out, lse, *grads, fb.fewbit_relative_bias_bwd(grads[3], table, bidirectional=True))

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step(5.0)
    torch.cuda.current_stream().wait_stream(side)
    graphs = []
    for cap in (5.0, 9.0):
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            held = step(cap)
        graphs.append((graph, held, cap))
    for seed in range(2):
        for x in docs:
            x.copy_(torch.randint(0, 3, x.shape, device="cuda", dtype=torch.int32).sort(1).values)
        table.normal_()
        for graph, _, _ in graphs:
            graph.replay()
        for _, held, cap in graphs:
            assert all(torch.equal(a, b) for a, b in zip(held, step(cap)))
    bias = fb.fewbit_relative_bias_fwd(table, 60, bidirectional=True)
    side.wait_stream(torch.cuda.current_stream())
    out, lse = fb.fewbit_attention_fwd(q, k, v, distance_bias=bias, stream=side)
    grads = fb.fewbit_attention_bwd(g, q, k, v, out, lse, distance_bias=bias, stream=side)
    db = fb.fewbit_relative_bias_bwd(grads[3], table, bidirectional=True, stream=side)
    side.synchronize()
    want = fb.fewbit_attention_bwd(g, q, k, v, *fb.fewbit_attention_fwd(q, k, v, distance_bias=bias), distance_bias=bias)
    assert all(torch.equal(a, b) for a, b in zip(grads, want)) and torch.equal(db, fb.fewbit_relative_bias_bwd(want[3], table, bidirectional=True))


@pytest.mark.gpu
@pytest.mark.parametrize("both", [False, True])
@pytest.mark.parametrize("dtype", [torch.float32, BF, HALF], ids=str)
def test_buckets(dtype, both):
    """Every distance's bucket against whole-number arithmetic; the gradient against 64-bit sums: (terms) 2^-24 of the magnitudes
    in 32 bits, and the type's rounding."""
    for buckets, most in ((32, 128), (4, 2), (4, 3), (6, 9), (16, 64), (32, 17), (64, 300), (10, 4096), (320, 800), (1024, 4096), (20, 1000)) + (((2, 2), (3, 2), (7, 50)) if not both else ()):
        if most <= (buckets // 2 if both else buckets) // 2:
            continue
        table = torch.randn(buckets, 5, device="cuda").to(dtype)
        bias = fb.fewbit_relative_bias_fwd(table, most, bidirectional=both)
        of = exact_buckets(buckets, most, both)
        assert torch.equal(bias, table.float()[of].T)
        g = torch.randn_like(bias)
        got = fb.fewbit_relative_bias_bwd(g, table, bidirectional=both)
        assert got.dtype == dtype and got.shape == table.shape
        want = torch.zeros(buckets, 5, dtype=torch.float64, device="cuda").index_add_(0, of, g.T.double())
        size = torch.zeros(buckets, 5, dtype=torch.float64, device="cuda").index_add_(0, of, g.T.double().abs())
        e = {torch.float32: 2.0 ** -24, BF: 2.0 ** -8, HALF: 2.0 ** -11}[dtype]
        assert ((got.double() - want).abs() <= e * want.abs() + (most / 32 + 8) * 2.0 ** -24 * size + (2.0 ** -25 if dtype == HALF else 0)).all()


def test_refusals_of_the_library():
    """No kernel is launched: every call ends at a check of the host."""
    lib = binding.load_library()
    some = ctypes.c_void_p(1 << 20)
    heads = ops._Heads((1 << 20), 64 * 2 * 100, 64 * 2, 64)

    def shape(causal=1, n=100, scale=0.125, h=2):
        return ops._AttentionShape(1, h, h, 64, n, n, 0, 0, None, None, causal, scale, 1)

    def fwd(s, **c):
        c = ops._AttentionScores(**c)
        x = ctypes.byref(heads)
        return lib.fewbit_attention_scores_fwd(ctypes.byref(s), ctypes.byref(c), x, x, x, x, None, None)

    at = 1 << 20
    assert fwd(shape(), cap=1.0) == 1                        # (only lse is missing)
    for cap in (-1.0, float("nan"), float("inf"), 3e38, 1e-42, 2.0 ** -61, 2.0 ** 61):
        assert fwd(shape(), cap=cap) == 1
    assert fwd(shape(), distance_bias=at, max_distance=0) == 1 and fwd(shape(), distance_bias=at, max_distance=4097) == 1
    assert fwd(shape(causal=0), prefix_lens=at) == 1
    assert fwd(shape(), q_documents=at) == 1 and fwd(shape(), k_documents=at) == 1
    for name in ("slopes", "distance_bias", "prefix_lens"):
        assert fwd(shape(), **{name: at + 2, "max_distance": 4}) == 3
    assert fwd(shape(), q_documents=at, k_documents=at + 1) == 3
    assert fwd(shape(n=(1 << 30) + 1), cap=1.0) == 6
    assert fwd(shape(h=70000), distance_bias=at, max_distance=4) == 6

    def bwd(s, c, db, ws=some, size=1 << 40, lse=some):
        x = ctypes.byref(heads)
        return lib.fewbit_attention_scores_bwd(ctypes.byref(s), ctypes.byref(c) if c else None, x, x, x, x, x, lse, x, x, x, db, ws, size, None)

    biased = ops._AttentionScores(distance_bias=at, max_distance=8)
    assert bwd(shape(), None, some) == 1 and bwd(shape(), ops._AttentionScores(cap=1.0), some) == 1
    assert bwd(shape(), biased, ctypes.c_void_p(at + 2)) == 3
    assert bwd(shape(), biased, some, ws=None) == 1 and bwd(shape(), biased, some, lse=None) == 1
    plain = lib.fewbit_attention_workspace_bytes(ctypes.byref(shape()))
    whole = lib.fewbit_attention_scores_workspace_bytes(ctypes.byref(shape()), ctypes.byref(biased), 1)
    assert plain == lib.fewbit_attention_scores_workspace_bytes(ctypes.byref(shape()), ctypes.byref(biased), 0) and whole > plain
    assert bwd(shape(), biased, some, size=whole - 1) == 5 and bwd(shape(), biased, None, size=plain - 1) == 5
    assert lib.fewbit_attention_scores_workspace_bytes(ctypes.byref(shape()), ctypes.byref(ops._AttentionScores(cap=-1.0)), 0) == 0

    def spread(table=some, buckets=32, h=4, most=128, both=0, dtype=0, bias=some):
        return lib.fewbit_relative_bias_fwd(table, buckets, h, most, both, dtype, bias, None)

    for bad in ({"buckets": 1}, {"buckets": 1025}, {"buckets": 2, "both": 1}, {"buckets": 33, "both": 1}, {"most": 16}, {"most": 4097}, {"h": -1}, {"dtype": 3},
                {"table": None}, {"bias": None}, {"buckets": 32, "both": 1, "most": 8}):
        assert spread(**bad) == 1
    assert spread(h=65536) == 6 and spread(h=0, table=None, bias=None) == 0
    assert spread(table=ctypes.c_void_p(at + 2)) == 3 and spread(table=ctypes.c_void_p(at + 1), dtype=1) == 3 and spread(bias=ctypes.c_void_p(at + 2)) == 3
    assert lib.fewbit_relative_bias_bwd(None, 32, 4, 128, 0, 0, some, None) == 1


@pytest.mark.gpu
def test_refusals_of_the_python_entry_points():
    q, k, v, _ = ta.make(2, 20, 30, 4, 2, 64, BF)
    i32 = {"dtype": torch.int32, "device": "cuda"}
    docs = {"q_documents": torch.zeros(2, 20, **i32), "k_documents": torch.zeros(2, 30, **i32)}
    for bad in ({"cap": -1.0}, {"cap": float("nan")}, {"slopes": torch.zeros(3, device="cuda")}, {"slopes": torch.zeros(4, device="cuda").half()}, {"slopes": torch.zeros(4)},
                {"distance_bias": torch.zeros(4, 8, device="cuda")}, {"distance_bias": torch.zeros(4, 1, device="cuda")}, {"distance_bias": torch.zeros(2, 9, device="cuda")},
                {"distance_bias": torch.zeros(9, 4, device="cuda").T}, {"distance_bias": torch.zeros(4, 8195, device="cuda")}, {"distance_bias": torch.zeros(4, 9, device="cuda").bfloat16()},
                {"prefix_lens": torch.zeros(2, **i32)}, {"prefix_lens": torch.zeros(3, **i32), "causal": True}, {"prefix_lens": torch.zeros(2, device="cuda"), "causal": True},
                {"q_documents": docs["q_documents"]}, {"k_documents": docs["k_documents"]}, {**docs, "k_documents": docs["q_documents"]},
                {**docs, "q_documents": docs["q_documents"].long()}, {**docs, "q_documents": torch.zeros(20, 2, **i32).T}):
        with pytest.raises(ValueError):
            fb.fewbit_attention_fwd(q, k, v, **bad)
    with pytest.raises(ValueError, match="slopes"):
        fb.fewbit_attention(q, k, v, slopes=torch.zeros(4, device="cuda", requires_grad=True))
    table = torch.zeros(32, 4, device="cuda")
    for call in (lambda: fb.fewbit_relative_bias_fwd(table, 0), lambda: fb.fewbit_relative_bias_fwd(table, 5000), lambda: fb.fewbit_relative_bias_fwd(table.T, 128),
                 lambda: fb.fewbit_relative_bias_fwd(table.double(), 128), lambda: fb.fewbit_relative_bias_fwd(table[0], 128),
                 lambda: fb.fewbit_relative_bias_bwd(torch.zeros(3, 9, device="cuda"), table), lambda: fb.fewbit_relative_bias_bwd(torch.zeros(4, 10, device="cuda"), table)):
        with pytest.raises(ValueError):
            call()
    with pytest.raises(fb.FewbitError):
        fb.fewbit_relative_bias_fwd(table, 16)


@pytest.mark.gpu
def test_gradients_through_autograd():
    """Table, bias and attention together, the bias shared by two layers and the table in bfloat16."""
    q, k, v, g = ta.make(2, 90, 90, 4, 2, 64, BF)
    q, k, v = (x.requires_grad_() for x in (q, k, v))
    table = torch.randn(16, 4, device="cuda").requires_grad_()
    bias = fb.fewbit_relative_bias(table, 30, bidirectional=True)
    a = fb.fewbit_attention(q, k, v, distance_bias=bias, cap=6.0)
    b = fb.fewbit_attention(q, k, v, distance_bias=bias, causal=True)
    (a * g).sum().backward(retain_graph=True)
    first = table.grad.clone()
    (b * g).sum().backward()
    of = exact_buckets(16, 30, True)
    spread = table.detach().double()[of].T.contiguous()
    want, tol = [0, 0], [0, 0]
    for i in range(2):
        for layer, mods in enumerate(({"cap": 6.0}, {})):
            r, _ = reference(*(x[i].detach().double() for x in (q, k, v, g)), layer == 1, 64 ** -0.5, bias=spread, **mods)
            want[layer] = want[layer] + torch.zeros(16, 4, dtype=torch.float64, device="cuda").index_add_(0, of, r["db"].T)
            tol[layer] = tol[layer] + torch.zeros(16, 4, dtype=torch.float64, device="cuda").index_add_(0, of, r["db_tol"].T)
    assert ((first.double() - want[0]).abs() <= tol[0]).all()
    assert ((table.grad.double() - want[0] - want[1]).abs() <= tol[0] + tol[1] + 2.0 ** -22 * table.grad.abs()).all()
    half = torch.randn(16, 4, device="cuda", dtype=BF).requires_grad_()
    fb.fewbit_attention(q, k, v, distance_bias=fb.fewbit_relative_bias(half, 30)).sum().backward()
    assert half.grad.dtype == BF and torch.isfinite(half.grad).all()
    # (no gradient of the bias wanted: none is computed)
    before = fb.fewbit_launch_count()
    fb.fewbit_attention(q, k, v, distance_bias=bias.detach()).sum().backward()
    assert fb.fewbit_launch_count() - before == 3


@pytest.mark.gpu
def test_masks_changed_before_the_backward_pass_are_an_error():
    q, k, v, _ = ta.make(1, 40, 40, 2, 1, 64, BF)
    q.requires_grad_()
    docs, prefix, slopes, bias = torch.zeros(1, 40, dtype=torch.int32, device="cuda"), torch.zeros(1, dtype=torch.int32, device="cuda"), torch.zeros(2, device="cuda"), torch.zeros(2, 9, device="cuda")
    for changed in (docs, prefix, slopes, bias):
        out = fb.fewbit_attention(q, k, v, causal=True, q_documents=docs, k_documents=docs, prefix_lens=prefix, slopes=slopes, distance_bias=bias)
        changed.add_(1)
        with pytest.raises(RuntimeError, match="modified by an inplace operation"):
            out.sum().backward()


@pytest.mark.gpu
def test_gradients_against_differences():
    """Central differences of the forward pass in binary16, in the directions of the gradients themselves: out is rounded to 2^-11, so
    a step that moves the sum by far more than its rounding (sqrt(n) 2^-11 of terms of size 1) is taken, and 3 % allowed for the curvature
    and the operands' own rounding."""
    q, k, v, g = ta.make(1, 60, 60, 2, 1, 64, HALF)
    mods = {"causal": True, "cap": 2.0, "prefix_lens": torch.tensor([20], dtype=torch.int32, device="cuda")}
    bias = torch.randn(2, 41, device="cuda") * 0.5
    value = lambda q, k, v, bias: (fb.fewbit_attention_fwd(q, k, v, distance_bias=bias, **mods)[0].double() * g.double()).sum()  # noqa: E731
    out, lse = fb.fewbit_attention_fwd(q, k, v, distance_bias=bias, **mods)
    grads = fb.fewbit_attention_bwd(g, q, k, v, out, lse, distance_bias=bias, **mods)
    for which, grad in enumerate(grads):
        args = [q, k, v, bias]
        step = 0.1 / float(grad.double().abs().max())
        up, down = list(args), list(args)
        up[which], down[which] = ((args[which].double() + s * step * grad.double()).to(args[which].dtype) for s in (1, -1))
        moved = ((up[which].double() - down[which].double()) * grad.double()).sum()
        assert abs(float(value(*up) - value(*down)) / float(moved) - 1) <= 0.03
