"""AdamW over many tensors against the formulas in 64 bits, and its refusals.

Tolerances (derived, u = 2^-24): a moment is two products and a sum of rounded constants, so its error is at most
8 u of the terms' magnitudes; the update adds a root, a product, a sum, a quotient and a product (another 16 u of its
magnitude), the parameter one product and one difference (4 u of it), then the rounding to its type.  An 8-bit moment is
one of the two float8 neighbours of the exact value / scale: within one float8 step (2^-3 of the value, at least 2^-9 of
the scale), up to the 32-bit errors above."""
import ctypes
import math

import pytest
import torch

import paper_2202_00441_b200 as fb
from paper_2202_00441_b200 import operators as ops

U = 2.0 ** -24
KW = dict(step=7, lr=3e-3, betas=(0.9, 0.99), eps=1e-8, weight_decay=0.1)
SIZES = [(1,), (255,), (256,), (257,), (3, 1000), (0,), (70000,), (513, 129)]


def reference(p, g, m, v, kw, scale=1.0):
    b1, b2 = kw["betas"]
    g = g * scale
    m, v = b1 * m + (1 - b1) * g, b2 * v + (1 - b2) * g * g
    upd = kw["lr"] * (m / (1 - b1 ** kw["step"])) / ((v / (1 - b2 ** kw["step"])).sqrt() + kw["eps"])
    return p * (1 - kw["lr"] * kw["weight_decay"]) - upd, m, v, upd


def make(sizes, dtype, bits, master, seed=0, offset=0, zero_block=False):
    gen = torch.Generator(device="cuda").manual_seed(seed)

    def new(shape, dt, std):
        n = math.prod(shape)
        return (torch.randn(n + offset, generator=gen, device="cuda") * std).to(dt)[offset:].view(shape)

    s = {"p": [], "g": [], "m": [], "v": [], "ms": [], "vs": [], "master": []}
    for shape in sizes:
        n = math.prod(shape)
        x = new(shape, torch.float32, 0.02)
        s["p"].append(x.to(dtype) if offset == 0 else torch.cat([x.new_zeros(offset), x.view(-1)]).to(dtype)[offset:].view(shape))
        s["master"].append(x.clone())
        g = new(shape, dtype, 1e-2)
        if zero_block:
            g.view(-1)[:256] = 0
        s["g"].append(g)
        m, r = new(shape, torch.float32, 1e-2), new(shape, torch.float32, 1e-2).abs()
        if zero_block:
            m.view(-1)[:256] = 0
            r.view(-1)[:256] = 0
        if bits == 32:
            s["m"].append(m), s["v"].append(r * r)
            continue
        for name, val in (("m", m), ("v", r)):
            blocks = -(-n // 256)
            pad = torch.zeros(blocks * 256, device="cuda")
            pad[:n] = val.view(-1)
            sc = pad.view(-1, 256).abs().amax(1) / 448 if n else pad.new_zeros(0)
            q = torch.where(sc > 0, 1 / sc, 0)[:, None] * pad.view(-1, 256) if n else pad.view(0, 256)
            codes = torch.zeros(n + offset, device="cuda").to(torch.float8_e4m3fn)
            codes[offset:] = q.reshape(-1)[:n].clamp(-448, 448).to(torch.float8_e4m3fn)
            s[name].append(codes[offset:].view(shape)), s[name + "s"].append(sc)
    return s


def handle(s, bits, master):
    return fb.fewbit_adamw_create(s["p"], s["m"], s["v"], *((s["ms"], s["vs"]) if bits == 8 else (None, None)),
                                  s["master"] if master else None)


def wide(codes, scale, n):
    return (codes.float().double().view(-1) * scale.double().repeat_interleave(256)[:n])


def check(before, s, bits, master, kw, scale=1.0):
    for i, p0 in enumerate(before["p"]):
        n = p0.numel()
        if n == 0:
            continue
        start = (before["master"] if master else before["p"])[i].double().view(-1)
        g = before["g"][i].double().view(-1)
        if bits == 8:
            m0 = wide(before["m"][i], before["ms"][i], n)
            v0 = wide(before["v"][i], before["vs"][i], n) ** 2
        else:
            m0, v0 = before["m"][i].double().view(-1), before["v"][i].double().view(-1)
        p, m, v, upd = reference(start, g, m0, v0, kw, scale)
        b1 = kw["betas"][0]
        m_err = 8 * U * (b1 * m0.abs() + (1 - b1) * (g * scale).abs())
        upd_err = 24 * U * upd.abs() + upd.abs() * m_err / m.abs().clamp_min(1e-300)
        got = (s["master"] if master else s["p"])[i].double().view(-1)
        bound = upd_err + 4 * U * p.abs()
        eps = {torch.float32: U, torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11}[s["p"][i].dtype]
        if master:
            assert ((got - p).abs() <= bound).all()
            assert torch.equal(s["p"][i], s["master"][i].to(s["p"][i].dtype))
        else:
            assert ((got - p).abs() <= bound + eps * 1.001 * p.abs() + 2.0 ** -25).all()
        if bits == 32:
            assert ((s["m"][i].double().view(-1) - m).abs() <= m_err + 1e-45).all()
            assert ((s["v"][i].double().view(-1) - v).abs() <= 8 * U * v + 1e-45).all()
            continue
        for name, val in (("m", m), ("v", v.sqrt())):
            sc = s[name + "s"][i].double()
            pad = torch.zeros(sc.numel() * 256, dtype=torch.float64, device="cuda")
            pad[:n] = val.abs()
            top = pad.view(-1, 256).amax(1)
            assert ((sc * 448 - top).abs() <= 1e-5 * top + 1e-38).all()
            each = sc.repeat_interleave(256)[:n]
            back = wide(s[name][i], s[name + "s"][i], n)
            step = torch.maximum(2.0 ** -9 * each, val.abs() / 8)
            assert ((back - val).abs() <= step * (1 + 1e-4)).all()
            if name == "v":
                assert (back[val > 0] > 0).all()


@pytest.mark.gpu
@pytest.mark.parametrize("bits", [32, 8])
@pytest.mark.parametrize("dtype,master", [(torch.float32, False), (torch.bfloat16, False), (torch.bfloat16, True),
                                          (torch.float16, True)])
@pytest.mark.parametrize("offset", [0, 1])
def test_step_matches_the_formula(dtype, master, bits, offset):
    s = make(SIZES, dtype, bits, master, offset=offset)
    before = {k: [t.clone() for t in v] for k, v in s.items()}
    h = handle(s, bits, master)
    launches = fb.fewbit_launch_count()
    fb.fewbit_adamw_step(h, s["g"], seed=123, **KW)
    assert fb.fewbit_launch_count() - launches == 1
    check(before, s, bits, master, KW)


@pytest.mark.gpu
@pytest.mark.parametrize("bits", [32, 8])
def test_hundreds_of_tensors_and_a_gradient_scale(bits):
    """More tensors than one launch describes, empty ones among them; results do not depend on where a launch ends."""
    sizes = [((37 * i) % 700,) for i in range(901)]
    s = make(sizes, torch.bfloat16, bits, True, seed=3)
    before = {k: [t.clone() for t in v] for k, v in s.items()}
    scale = torch.tensor(0.125, device="cuda")
    launches = fb.fewbit_launch_count()
    fb.fewbit_adamw_step(handle(s, bits, True), s["g"], seed=5, grad_scale=scale, **KW)
    assert fb.fewbit_launch_count() - launches == 3
    check(before, s, bits, True, KW, 0.125)


@pytest.mark.gpu
def test_other_stream_and_repeatability():
    s = make([(5000,), (77, 13)], torch.float32, 8, False, seed=9)
    t = {k: [x.clone() for x in v] for k, v in s.items()}
    fb.fewbit_adamw_step(handle(s, 8, False), s["g"], seed=11, **KW)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    fb.fewbit_adamw_step(handle(t, 8, False), t["g"], seed=11, stream=side, **KW)
    torch.cuda.synchronize()
    for k in ("p", "ms", "vs"):
        assert all(torch.equal(a, b) for a, b in zip(s[k], t[k]))
    for k in ("m", "v"):
        assert all(torch.equal(a.view(torch.uint8), b.view(torch.uint8)) for a, b in zip(s[k], t[k]))


@pytest.mark.gpu
def test_rounding_is_unbiased_over_seeds():
    """The mean over 512 seeds of a rounded moment: with a step d between its neighbours the mean's standard deviation is
    at most d / 2 / sqrt(512); the bound is six of them plus the 2^-16 step of the random numbers."""
    n, seeds = 4096, 512
    base = make([(n,)], torch.float32, 8, False, seed=21)
    mean = {"m": 0, "v": 0}
    for seed in range(seeds):
        s = {k: [x.clone() for x in v] for k, v in base.items()}
        fb.fewbit_adamw_step(handle(s, 8, False), s["g"], seed=seed * 2654435761 % 2 ** 32, **KW)
        for k in mean:
            mean[k] = mean[k] + wide(s[k][0], s[k + "s"][0], n) / seeds
    m0, v0 = wide(base["m"][0], base["ms"][0], n), wide(base["v"][0], base["vs"][0], n) ** 2
    _, m, v, _ = reference(base["p"][0].double(), base["g"][0].double(), m0, v0, KW)
    for k, val in (("m", m), ("v", v.sqrt())):
        each = s[k + "s"][0].double().repeat_interleave(256)[:n]
        step = torch.maximum(2.0 ** -9 * each, 2.0 ** torch.floor(torch.log2(val.abs() / each)) * each / 8)
        assert ((mean[k] - val).abs() <= step * (3 / math.sqrt(seeds) + 2.0 ** -15)).all()


@pytest.mark.gpu
def test_zero_blocks_and_non_finite_values():
    s = make([(1024,)], torch.float32, 8, False, zero_block=True)
    s["g"][0][300] = float("nan")
    s["g"][0][600] = float("inf")
    fb.fewbit_adamw_step(handle(s, 8, False), s["g"], seed=1, **KW)
    m = wide(s["m"][0], s["ms"][0], 1024)
    assert (m[:256] == 0).all() and float(s["ms"][0][0]) == 0
    assert torch.isfinite(s["p"][0][:256]).all()              # 0 / (0 + eps): no update but the decay
    assert m[256:768].isnan().all() and m[768:].isfinite().all()
    assert s["p"][0][300].isnan() and s["p"][0][301].isfinite()


@pytest.mark.gpu
def test_binding_refuses_what_does_not_match():
    s = make([(300,)], torch.float32, 8, False)
    h = handle(s, 8, False)
    with pytest.raises(ValueError):
        fb.fewbit_adamw_step(h, [], **KW)
    with pytest.raises(ValueError):
        fb.fewbit_adamw_step(h, [s["g"][0].half()], **KW)
    with pytest.raises(ValueError):
        fb.fewbit_adamw_step(h, [torch.zeros(600, device="cuda")[::2]], **KW)
    with pytest.raises(ValueError):
        fb.fewbit_adamw_create(s["p"], s["m"], s["v"], s["ms"], [x[:1] for x in s["vs"]])
    with pytest.raises(ValueError):
        fb.fewbit_adamw_create(s["p"], s["m"], s["v"], s["ms"], s["vs"], s["p"])
    with pytest.raises(fb.FewbitError):
        fb.fewbit_adamw_step(h, s["g"], **(KW | {"step": 0}))


def test_library_refusals_need_no_gpu():
    lib = fb.load_library()
    A = 1 << 20
    T = ops._AdamWTensor

    def call(t, o=None, grad=A, count=1):
        opt = dict(lr=1e-3, beta1=0.9, beta2=0.99, eps=1e-8, weight_decay=0.0, step=1, state_bits=8, dtype=1) | (o or {})
        arr = (T * 2)(t, t)
        grads = (ctypes.c_void_p * 2)(grad, grad)
        return lib.fewbit_adamw_step(arr, grads, count, ctypes.byref(ops._AdamWOptions(**opt)), None)

    good = T(A, A, A, A, A, A, 100)
    for o in ({"step": 0}, {"beta1": 1.0}, {"beta2": -0.1}, {"eps": float("nan")}, {"lr": float("inf")}, {"weight_decay": -1.0},
              {"state_bits": 4}, {"dtype": 9}, {"lr": -1e-3}, {"dtype": 0}):
        assert call(good, o) == 1, o
    assert call(T(None, A, A, A, A, A, 100)) == 1 and call(good, grad=None) == 1
    assert call(T(A, A, A, None, A, A, 100)) == 1
    assert call(T(A + 1, A, A, A, A, A, 100)) == 3 and call(T(A, A, A, A + 2, A, A, 100)) == 3
    assert call(T(A, A + 2, A, None, None, A, 100), {"state_bits": 32}) == 3
    assert call(T(A, A, A, A, A, A, 1 << 39)) == 6
    assert call(good, count=-1) == 1 and call(good, count=0) == 0
    assert call(T(None, None, None, None, None, None, 0)) == 0
    assert lib.fewbit_adamw_step(None, None, 1, None, None) == 1
