"""AdamW at its edges: blocks of the smallest magnitudes, the noise of stochastic rounding over places, launches and steps, and
the handles that an optimizer keeps."""
import math

import pytest
import torch

import paper_2202_00441_b200 as fb
import test_adamw as tw
from paper_2202_00441_b200 import optim

WEYL = 0x9E3779B1                                                 # the noise of a place is a hash of place * WEYL + seed


# ---- blocks of tiny values ----------------------------------------------------------------------------------------------------
@pytest.mark.gpu
@pytest.mark.parametrize("top", [2.0 ** -118, 2.0 ** -119.5, 2.0 ** -122, 1e-37, 2.0 ** -126])
def test_blocks_of_tiny_moments_keep_their_values(top):
    """Moments with zero gradients decay through these sizes.  The scale of a block is top / 448, a subnormal here: its step of
    2^-149 is at most 2^-14.1 of it (2^-126 / 448 = 2^-134.8), so a value is off by one float8 step or by that."""
    n = 512
    gen = torch.Generator(device="cuda").manual_seed(4)
    m = torch.randn(n, generator=gen, device="cuda").clamp(-3, 3) / 3 * 0.9 * top
    m[0], m[1::5] = top, 0.0
    m[256] = -top
    p = torch.zeros(n, device="cuda")                             # moments from a gradient alone
    codes = [torch.zeros(n, device="cuda").to(torch.float8_e4m3fn) for _ in range(2)]
    scales = [torch.zeros(2, device="cuda") for _ in range(2)]
    g = (m.double() / 0.5).float()
    h = fb.fewbit_adamw_create([p], codes[:1], codes[1:], scales[:1], scales[1:])
    fb.fewbit_adamw_step(h, [g], step=1, lr=0.0, betas=(0.5, 0.5), eps=1e-8, seed=77)
    want = 0.5 * g.double()
    back = tw.wide(codes[0], scales[0], n)
    each = scales[0].double().repeat_interleave(256)
    assert ((scales[0].double() * 448 - top).abs() <= 2.0 ** -13 * top).all()
    step = torch.maximum(2.0 ** -9 * each, want.abs() / 8)
    assert ((back - want).abs() <= step * (1 + 2.0 ** -12) + 2.0 ** -13 * want.abs()).all()
    assert (back[want == 0] == 0).all()
    assert ((back[[0, 256]] - want[[0, 256]]).abs() <= 2.0 ** -13 * top).all()


@pytest.mark.gpu
def test_blocks_below_the_normal_numbers_read_back_as_zero():
    g = torch.full((256,), 2.0 ** -127, device="cuda")
    codes = [torch.zeros(256, device="cuda").to(torch.float8_e4m3fn) for _ in range(2)]
    scales = [torch.zeros(1, device="cuda") for _ in range(2)]
    h = fb.fewbit_adamw_create([torch.zeros(256, device="cuda")], codes[:1], codes[1:], scales[:1], scales[1:])
    fb.fewbit_adamw_step(h, [g], step=1, lr=0.0, betas=(0.5, 0.5), eps=1e-8, seed=1)
    assert float(scales[0]) == 0 and (tw.wide(codes[0], scales[0], 256) == 0).all()


# ---- noise ------------------------------------------------------------------------------------------------------------------
@pytest.mark.gpu
def test_noise_goes_on_over_the_ends_of_launches():
    """901 tensors in three launches give the same codes as one tensor with the same values at the same places."""
    sizes = [((37 * i) % 700,) for i in range(901)]
    s = tw.make(sizes, torch.float32, 8, False, seed=31)
    blocks = [-(-n // 256) for (n,) in sizes]
    total = sum(blocks) * 256
    flat = {k: torch.zeros(total, device="cuda") for k in ("p", "g")}
    flat |= {k: torch.zeros(total, device="cuda").to(torch.float8_e4m3fn) for k in ("m", "v")}
    flat |= {k: torch.cat(s[k]) for k in ("ms", "vs")}
    at = [256 * sum(blocks[:i]) for i in range(len(sizes))]
    for k in ("p", "g", "m", "v"):
        for a, (n,), x in zip(at, sizes, s[k]):
            flat[k].view(torch.uint8 if k in "mv" else torch.float32)[a:a + n] = x.view(torch.uint8 if k in "mv" else torch.float32)
    fb.fewbit_adamw_step(tw.handle(s, 8, False), s["g"], seed=99, **tw.KW)
    one = fb.fewbit_adamw_create([flat["p"]], [flat["m"]], [flat["v"]], [flat["ms"]], [flat["vs"]])
    fb.fewbit_adamw_step(one, [flat["g"]], seed=99, **tw.KW)
    for k in ("m", "v"):
        whole = flat[k].view(torch.uint8)
        assert all(torch.equal(whole[a:a + n], x.view(torch.uint8)) for a, (n,), x in zip(at, sizes, s[k]))
    assert torch.equal(flat["ms"], torch.cat(s["ms"])) and torch.equal(flat["vs"], torch.cat(s["vs"]))


@pytest.mark.gpu
def test_rounding_is_unbiased_over_unrelated_seeds():
    """The mean over 512 seeds that are no multiples of one another: with a step d between its neighbours the mean's standard
    deviation is at most d / 2 / sqrt(512); the bound is six of them plus the 2^-16 step of the random numbers."""
    n, seeds = 4096, 512
    base = tw.make([(n,)], torch.float32, 8, False, seed=22)
    drawn = torch.randint(0, 2 ** 32, (seeds,), generator=torch.Generator().manual_seed(5)).tolist()
    mean = {"m": 0, "v": 0}
    for seed in drawn:
        s = {k: [x.clone() for x in v] for k, v in base.items()}
        fb.fewbit_adamw_step(tw.handle(s, 8, False), s["g"], seed=seed, **tw.KW)
        for k in mean:
            mean[k] = mean[k] + tw.wide(s[k][0], s[k + "s"][0], n) / seeds
    m0, v0 = tw.wide(base["m"][0], base["ms"][0], n), tw.wide(base["v"][0], base["vs"][0], n) ** 2
    _, m, v, _ = tw.reference(base["p"][0].double(), base["g"][0].double(), m0, v0, tw.KW)
    for k, val in (("m", m), ("v", v.sqrt())):
        each = s[k + "s"][0].double().repeat_interleave(256)[:n]
        step = torch.maximum(2.0 ** -9 * each, 2.0 ** torch.floor(torch.log2(val.abs() / each)) * each / 8)
        assert ((mean[k] - val).abs() <= step * (3 / math.sqrt(seeds) + 2.0 ** -15)).all()


class _Recorder:
    """Stands for fewbit_adamw_create and fewbit_adamw_step: what an optimizer asks of them."""

    def __init__(self, monkeypatch):
        self.created, self.seeds = 0, []
        monkeypatch.setattr(optim, "fewbit_adamw_create", self.create)
        monkeypatch.setattr(optim, "fewbit_adamw_step", lambda h, grads, *, seed, **kw: self.seeds.append(seed))

    def create(self, *lists):
        self.created += 1
        return object()


class _CpuAdamW(fb.FewBitAdamW):
    def add_param_group(self, group):                            # without the check for CUDA tensors
        torch.optim.Optimizer.add_param_group(self, group)


def _steps(opt, params, count, missing=()):
    for step in range(count):
        for i, p in enumerate(params):
            p.grad = None if (step, i) in missing else torch.ones_like(p)
        opt.step()


def test_steps_of_the_optimizer_do_not_share_their_noise(monkeypatch):
    """Two seeds s and t give the same noise field, moved by (t - s) / WEYL mod 2^32 places.  Steps that follow one another, and
    groups and types within a step, have to lie far apart: 4096 places, which chance leaves in 2 of 10^6 pairs."""
    rec = _Recorder(monkeypatch)
    params = [torch.nn.Parameter(torch.zeros(8, dtype=t)) for t in (torch.float32, torch.bfloat16, torch.float32)]
    opt = _CpuAdamW([{"params": params[:2]}, {"params": params[2:]}], seed=5)
    _steps(opt, params, 300)
    assert len(rec.seeds) == 900 and all(0 <= s < 2 ** 32 for s in rec.seeds)
    back = pow(WEYL, -1, 2 ** 32)
    for near in range(1, 7):                                     # the same and the next two steps
        for s, t in zip(rec.seeds, rec.seeds[near:]):
            shift = (t - s) * back % 2 ** 32
            assert min(shift, 2 ** 32 - shift) > 4096
    again = _Recorder(monkeypatch)
    _steps(_CpuAdamW([{"params": params[:2]}, {"params": params[2:]}], seed=5), params, 10)
    assert again.seeds == rec.seeds[:30]
    other = _Recorder(monkeypatch)
    _steps(_CpuAdamW([{"params": params[:2]}, {"params": params[2:]}], seed=6), params, 10)
    assert not set(other.seeds) & set(again.seeds)


# ---- handles ------------------------------------------------------------------------------------------------------------------
def test_parameters_a_step_apart_keep_their_handles(monkeypatch):
    rec = _Recorder(monkeypatch)
    params = [torch.nn.Parameter(torch.zeros(8)) for _ in range(3)]
    opt = _CpuAdamW(params)
    _steps(opt, params, 3, missing={(1, 2)})                     # the last parameter falls a step behind
    made = rec.created
    _steps(opt, params, 20)
    assert rec.created <= made + 1                               # (two handles for the two of them, from then on)


@pytest.mark.gpu
@pytest.mark.parametrize("bits", [8, 32])
def test_a_handle_follows_its_tensors(bits):
    """Other memory put under a parameter and its state: the next step works there, and nothing is written where they lay."""
    s, t = (tw.make([(700,), (300,)], torch.bfloat16, bits, True, seed=41) for _ in range(2))
    h, other = tw.handle(s, bits, True), tw.handle(t, bits, True)
    names = [k for k in s if k != "g" and s[k]]
    left = {k: [x.detach() for x in s[k]] for k in names}        # keeps the old memory
    for k in names:
        for x in s[k]:
            x.data = x.data.clone()
    before = {k: [x.clone() for x in left[k]] for k in names}
    fb.fewbit_adamw_step(h, s["g"], seed=7, **tw.KW)
    fb.fewbit_adamw_step(other, t["g"], seed=7, **tw.KW)

    def same(a, b):
        return torch.equal(a.view(torch.uint8), b.view(torch.uint8))

    for k in names:
        assert all(same(a, b) for a, b in zip(s[k], t[k])), k
        assert all(same(a, b) for a, b in zip(left[k], before[k])), k
    s["p"][0].data = s["p"][0].data[:100].clone()
    with pytest.raises(ValueError):
        fb.fewbit_adamw_step(h, s["g"], seed=8, **tw.KW)
