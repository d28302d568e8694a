"""Dropout from a counter, and the norm of the residual stream, against the formulas in 64 bits; refusals.

Tolerances (derived).  e = half a step of the type (2^-8, 2^-11, 2^-24), t = its smallest step's half (binary16: 2^-25).
 dropout   one product and one sum in 32 bits, one rounding: (e + 2^-23) (|r| + |x| / (1 - p)); without a residual in
           binary32 the product alone, which is the same everywhere: equal.
 h         the same.  y = h s w: a thread adds at most 32 squares, then 9 pairs: s^2 is off by 41 roundings of 2^-24 at most, s by
           half of that and rsqrtf's two units, and two products: below 2^-18 together.
 gradient  grad_h + s (g w - u m), m = mean(g w u): its terms are each off by less than 2^-17 of their magnitudes.
 grad_w    sums of one row after another in 32 bits, at most `rows` of them and then 37: (rows + 40) 2^-24 sum |g u|, and u's 2^-18.
 8 bits    half a step of the code, 2^-4 relative or 2^-10 scales, and y's own 2^-17; the scale 2^-17."""
import ctypes

import numpy as np
import pytest
import torch

import paper_2202_00441_b200 as fb
from paper_2202_00441_b200 import binding, operators as ops

E = {torch.float32: 2.0 ** -24, torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11}
TINY = {torch.float32: 0.0, torch.bfloat16: 0.0, torch.float16: 2.0 ** -25}
TYPES = [torch.float32, torch.bfloat16, torch.float16]


def philox(c, k):
    """One block by the definition: four counters and two keys of 32 bits (arrays of uint64)."""
    c, k = [np.asarray(x, dtype=np.uint64) for x in c], [int(x) for x in k]
    low = np.uint64(0xFFFFFFFF)
    for _ in range(10):
        a, b = c[0] * np.uint64(0xD2511F53), c[2] * np.uint64(0xCD9E8D57)
        c = [(b >> np.uint64(32)) ^ c[1] ^ np.uint64(k[0]), b & low, (a >> np.uint64(32)) ^ c[3] ^ np.uint64(k[1]), a & low]
        k = [(k[0] + 0x9E3779B9) & 0xFFFFFFFF, (k[1] + 0xBB67AE85) & 0xFFFFFFFF]
    return c


def kept(shape, p, seed, place, first=0):
    """The mask of a tensor's elements from `first` (a multiple of 4) on."""
    n = int(np.prod(shape))
    group = np.arange(first // 4, first // 4 + (n + 3) // 4, dtype=np.uint64)
    words = np.stack(philox((group & np.uint64(0xFFFFFFFF), group >> np.uint64(32), np.full_like(group, place), np.zeros_like(group)),
                            (seed & 0xFFFFFFFF, seed >> 32)), 1).reshape(-1)[:n]
    return torch.from_numpy((words >= round(p * 2 ** 32)).reshape(shape))


def test_the_oracle_gives_the_generators_published_words():
    """Known answers of Philox4x32-10 as its authors publish them."""
    for c, k, words in ((4 * [0], 2 * [0], [0x6627e8d5, 0xe169c58d, 0xbc57ac4c, 0x9b00dbd8]),
                        (4 * [0xffffffff], 2 * [0xffffffff], [0x408f276d, 0x41c83b0e, 0xa20bc7c6, 0x6d5451fd]),
                        ([0x243f6a88, 0x85a308d3, 0x13198a2e, 0x03707344], [0xa4093822, 0x299f31d0], [0xd16cfe09, 0x94fdcceb, 0x5001e420, 0x24126ea1])):
        assert [int(x) for x in philox(c, k)] == words


def test_refusals_of_the_library():
    """No kernel is launched: every call ends at a check of the host."""
    lib = binding.load_library()
    some = ctypes.c_void_p(1 << 20)

    def drop(p=0.1, seed_device=None):
        return ops._DropoutOptions(p, 1, seed_device, 0)

    def fwd(x=some, r=None, y=some, n=8, dtype=0, o=None):
        return lib.fewbit_dropout_fwd(x, r, y, n, dtype, ctypes.byref(o or drop()), None)

    assert fwd(n=0) == 0 and fwd(x=None, y=None, n=0) == 0
    assert lib.fewbit_dropout_fwd(some, None, some, 8, 0, None, None) == 1
    assert fwd(x=None) == 1 and fwd(y=None) == 1 and fwd(dtype=3) == 1 and fwd(dtype=-1) == 1
    for p in (-0.1, 1.0, 2.0, float("nan"), float("inf")):
        assert fwd(o=drop(p)) == 1
    assert fwd(x=ctypes.c_void_p((1 << 20) + 2)) == 3 and fwd(r=ctypes.c_void_p((1 << 20) + 1), dtype=1) == 3
    assert fwd(o=drop(seed_device=4)) == 3
    assert fwd(n=1 << 60) == 6
    assert lib.fewbit_dropout_bwd(None, some, 8, 0, ctypes.byref(drop()), None) == 1

    def shape(rows=4, width=64, weight=None, eps=1e-6, dtype=0, p=0.0):
        return ops._NormShape(rows, width, weight, eps, dtype, drop(p))

    def norm(s, x=some, r=None, h=None, y=some, scale=None, bits=0):
        return lib.fewbit_add_rms_norm_fwd(ctypes.byref(s) if s else None, x, r, h, y, scale, bits, None)

    assert norm(None) == 1 and norm(shape(rows=-1)) == 1 and norm(shape(width=-1)) == 1 and norm(shape(dtype=7)) == 1
    assert norm(shape(eps=-1.0)) == 1 and norm(shape(eps=float("nan"))) == 1 and norm(shape(eps=float("inf"))) == 1 and norm(shape(p=1.0)) == 1
    assert norm(shape(width=16385)) == 2 and norm(shape(rows=1 << 31)) == 6
    assert norm(shape(), x=None) == 1 and norm(shape(), y=None) == 1
    assert norm(shape(), bits=4) == 1 and norm(shape(), bits=8) == 1 and norm(shape(), scale=some) == 1
    assert norm(shape(weight=2)) == 3 and norm(shape(), x=ctypes.c_void_p((1 << 20) + 2)) == 3
    assert norm(shape(), scale=ctypes.c_void_p((1 << 20) + 2), bits=8) == 3
    assert norm(shape(rows=0)) == 0 and norm(shape(width=0)) == 0

    def bwd(s, gy=some, gh=None, h=some, gx=some, gr=None, gw=None, ws=None, size=0):
        return lib.fewbit_add_rms_norm_bwd(ctypes.byref(s), gy, gh, h, gx, gr, gw, ws, size, None)

    assert bwd(shape(), gy=None) == 1 and bwd(shape(), h=None) == 1 and bwd(shape(), gw=some) == 1
    assert bwd(shape(), gw=ctypes.c_void_p((1 << 20) + 2), ws=some) == 3 and bwd(shape(), gw=some, ws=ctypes.c_void_p((1 << 20) + 8)) == 3
    assert bwd(shape(width=20000)) == 2 and bwd(shape(rows=0)) == 0
    assert lib.fewbit_add_rms_norm_workspace_bytes(ctypes.byref(shape(width=20000))) == 0


def new(shape, dtype, seed, size=1.0, offset=0):
    """A tensor of a shape, `offset` elements into its buffer."""
    gen = torch.Generator(device="cuda").manual_seed(seed)
    n = int(np.prod(shape))
    flat = torch.zeros(n + offset, dtype=dtype, device="cuda")
    flat[offset:] = (torch.randn(n, generator=gen, device="cuda") * size).to(dtype)
    return flat[offset:].view(shape)


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", TYPES, ids=str)
@pytest.mark.parametrize("n,offset", [(1, 0), (3, 1), (8, 0), (31, 0), (1000, 2), (8192, 0), (8193, 0), (8200, 8), (65536 + 5, 3), (300001, 0)])
def test_dropout(dtype, n, offset):
    x, r, g = new((n,), dtype, 1, 2.0, offset), new((n,), dtype, 2, 1.0, offset), new((n,), dtype, 3, 1.0, offset)
    for p, seed, place in ((0.0, 1, 0), (0.1, 0x123456789abcdef0, 7), (0.5, (1 << 64) - 1, (1 << 32) - 1), (0.999, 3, 1)):
        mask = kept((n,), p, seed, place).cuda()
        scale = torch.tensor(1 / (1 - p), dtype=torch.float32, device="cuda")
        want = torch.where(mask, x.float() * scale, 0.0).to(dtype)
        kw = {"p": p, "seed": seed, "place": place}
        assert torch.equal(fb.fewbit_dropout_fwd(x, **kw), want)
        assert torch.equal(fb.fewbit_dropout_bwd(g, **kw), torch.where(mask, g.float() * scale, 0.0).to(dtype))
        got = fb.fewbit_dropout_fwd(x, residual=r, **kw)
        exact = r.double() + torch.where(mask, x.double() / (1 - p), 0.0)
        assert ((got.double() - exact).abs() <= (E[dtype] + 2.0 ** -23) * (r.double().abs() + x.double().abs() / (1 - p)) + TINY[dtype]).all()
        for out in ("x", "r"):
            a, b = x.clone(), r.clone()
            to = {"x": a, "r": b}[out]
            assert fb.fewbit_dropout_fwd(a, residual=b, out=to, **kw) is to and torch.equal(to, got)
        assert fb.fewbit_dropout_bwd(g, out=g.clone(), **kw).equal(fb.fewbit_dropout_bwd(g, **kw))


@pytest.mark.gpu
def test_dropout_of_what_is_not_finite():
    """What is dropped is 0 whatever it held; what is kept stays what it was."""
    x = torch.tensor([float("inf"), float("nan"), -float("inf"), 1.0] * 64, device="cuda")
    mask = kept((256,), 0.5, 9, 0).cuda()
    y = fb.fewbit_dropout_fwd(x, 0.5, seed=9)
    assert torch.equal(torch.isnan(y), torch.isnan(x) & mask) and torch.equal(torch.isinf(y), torch.isinf(x) & mask) and (y[~mask] == 0).all()


@pytest.mark.gpu
def test_dropout_keeps_the_share_it_says():
    """8 million draws: five standard deviations; two places have unrelated masks."""
    n, p = 1 << 23, 0.3
    x = torch.ones(n, device="cuda")
    masks = [fb.fewbit_dropout_fwd(x, p, seed=5, place=i) != 0 for i in (0, 1)]
    for m in masks:
        assert abs(m.double().mean().item() - (1 - p)) <= 5 * (p * (1 - p) / n) ** 0.5
    both = (masks[0] & masks[1]).double().mean().item()
    assert abs(both - (1 - p) ** 2) <= 5 * (0.25 / n) ** 0.5


@pytest.mark.gpu
def test_dropout_past_32_bits_of_elements():
    n, tail = (1 << 32) + 4104, 4096
    x = torch.ones(n, dtype=torch.bfloat16, device="cuda")
    y = fb.fewbit_dropout_fwd(x, 0.25, seed=77, place=2, out=x)
    for first in (0, (1 << 32) - 2048, n - tail):
        assert torch.equal(y[first:first + tail] != 0, kept((tail,), 0.25, 77, 2, first).cuda())


def norm_reference(x, r, w, eps, p, mask):
    """64 bits: h, y, u, s."""
    h = torch.where(mask, x / (1 - p), 0.0) + (0 if r is None else r)
    s = (h.square().mean(-1, keepdim=True) + eps).rsqrt()
    return h, h * s * (1 if w is None else w), h * s, s


CASES = [
    # rows, width, offset in elements, p, residual, weight
    (1, 1, 0, 0.0, True, True), (3, 3, 0, 0.1, True, True), (70, 4, 0, 0.0, False, True), (5, 8, 0, 0.5, True, False), (2, 20, 0, 0.1, True, True),
    (9, 31, 1, 0.1, True, True), (17, 64, 0, 0.0, True, True), (33, 333, 0, 0.2, True, True), (4, 512, 0, 0.1, False, False), (5, 640, 0, 0.0, True, True),
    (300, 1000, 4, 0.1, True, True), (2, 1288, 8, 0.0, True, True), (3, 2052, 0, 0.1, True, True), (700, 4096, 0, 0.1, True, True), (2, 8191, 3, 0.1, True, True),
    (2, 8192, 0, 0.0, True, True), (3, 8200, 0, 0.1, True, True), (2, 16383, 0, 0.1, True, True), (1, 16384, 0, 0.1, True, True), (1300, 16384, 0, 0.0, True, True),
    (40000, 48, 0, 0.1, True, True), (5000, 5, 0, 0.2, True, True), (3000, 256, 0, 0.1, True, True), (1000, 509, 0, 0.1, True, True), (20000, 1026, 0, 0.0, True, True),
    (700, 4099, 0, 0.1, True, True), (500, 8197, 0, 0.0, True, True), (9, 16377, 0, 0.1, True, True), (3, 2049, 8, 0.1, True, False),
]


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", TYPES, ids=str)
@pytest.mark.parametrize("case", CASES, ids=lambda c: "x".join(map(str, c)))
def test_norm(case, dtype):
    rows, width, offset, p, with_r, with_w = case
    e, t, eps, seed, place = E[dtype], TINY[dtype], 1e-6, 0x1357924680abcdef, 11
    x, r = new((rows, width), dtype, 1, 1.0, offset), new((rows, width), dtype, 2, 2.0, offset) if with_r else None
    w = new((width,), torch.float32, 3, 0.3, offset) + 1 if with_w else None
    if with_w and offset:
        w = torch.cat([torch.zeros(1, device="cuda"), w])[1:]     # 4 bytes from an even address
    kw = {"eps": eps, "p": p, "seed": seed, "place": place}
    mask = kept((rows, width), p, seed, place).cuda() if p else torch.ones(rows, width, dtype=torch.bool, device="cuda")
    wd = None if w is None else w.double()
    h, y, u, s = norm_reference(x.double(), None if r is None else r.double(), wd, eps, p, mask)

    got_y, got_h = fb.fewbit_add_rms_norm_fwd(x, r, w, **kw)
    mag = x.double().abs() / (1 - p) + (0 if r is None else r.double().abs())
    assert ((got_h.double() - h).abs() <= (e + 2.0 ** -23) * mag + t).all()
    # (one element's own cancellation in h moves its u too)
    assert ((got_y.double() - y).abs() <= (e + 2.0 ** -18) * y.abs() + 2.0 ** -22 * mag * s * (1 if w is None else wd.abs()) + t).all()
    if r is None and not p:
        assert got_h is x or got_h.data_ptr() == x.data_ptr()

    codes, scale, h8 = fb.fewbit_add_rms_norm_fwd(x, r, w, bits=8, **kw)
    assert codes.dtype == torch.float8_e4m3fn and scale.shape == (rows,) and torch.equal(h8, got_h)
    top = y.abs().amax(-1)
    assert ((scale.double() - top / 448).abs() <= 2.0 ** -16 * top / 448).all()
    sc = scale.double()[:, None]
    assert ((codes.double() * sc - y).abs() <= torch.maximum(2.0 ** -4 * y.abs(), 2.0 ** -10 * sc) + 2.0 ** -16 * y.abs() + 2.0 ** -20 * mag * s * (1 if w is None else wd.abs())).all()

    gy, gh = new((rows, width), dtype, 4, 1.0, offset), new((rows, width), dtype, 5, 0.5, offset)
    hd = got_h.double()
    s = (hd.square().mean(-1, keepdim=True) + eps).rsqrt()
    u, g = hd * s, gy.double() * (1 if w is None else wd)
    back = (g * u).mean(-1, keepdim=True)
    for other in (None, gh):
        gx, gr, gw = fb.fewbit_add_rms_norm_bwd(gy, other, got_h, w, **kw)
        o = 0 if other is None else other.double()
        want = o + s * (g - u * back)
        bound = e * want.abs() + t + 2.0 ** -17 * (abs(o) + s * g.abs() + s * u.abs() * (g * u).abs().mean(-1, keepdim=True))
        assert ((gr.double() - want).abs() <= bound).all()
        assert ((gx.double() - torch.where(mask, want / (1 - p), 0.0)).abs() <= torch.where(mask, (bound + 2.0 ** -22 * want.abs()) / (1 - p) + t, 0.0)).all()
        if not p:
            assert gx is gr or gx.data_ptr() == gr.data_ptr()
        terms = (gy.double() * u).abs().sum(0)
        assert gw.dtype == torch.float32
        assert ((gw.double() - (gy.double() * u).sum(0)).abs() <= ((rows + 40) * 2.0 ** -24 + 2.0 ** -18) * terms).all()
    again = fb.fewbit_add_rms_norm_bwd(gy, gh, got_h, w, **kw)
    assert torch.equal(again[0], gx) and torch.equal(again[1], gr) and torch.equal(again[2], gw)
    only = fb.fewbit_add_rms_norm_bwd(gy, gh, got_h, w, residual_grad=False, weight_grad=False, **kw)
    assert only[1] is None and only[2] is None and torch.equal(only[0], gx)
    only = fb.fewbit_add_rms_norm_bwd(gy, gh, got_h, w, x_grad=False, **kw)
    assert only[0] is None and torch.equal(only[1], gr) and torch.equal(only[2], gw)


@pytest.mark.gpu
def test_norm_rows_that_are_empty_zero_or_not_finite():
    for shape in ((0, 64), (3, 0), (0, 0)):
        x = torch.empty(shape, device="cuda", dtype=torch.bfloat16)
        y, h = fb.fewbit_add_rms_norm_fwd(x, x)
        assert y.shape == shape and h.shape == shape
        codes, scale, _ = fb.fewbit_add_rms_norm_fwd(x, x, bits=8)
        assert codes.shape == shape and (scale == 0).all()
        gx, gr, gw = fb.fewbit_add_rms_norm_bwd(x, None, x)
        assert gx.shape == shape and gw.shape == (shape[1],) and (gw == 0).all()
    x = torch.randn(5, 40, device="cuda")
    x[1] = 0
    x[2, 7] = float("nan")
    x[3, 9] = float("inf")
    x[4] *= 1e-30
    codes, scale, _ = fb.fewbit_add_rms_norm_fwd(x, eps=1e-6, bits=8)
    y, _ = fb.fewbit_add_rms_norm_fwd(x, eps=1e-6)
    back = codes.float() * scale[:, None]
    assert torch.isnan(back[2:4]).all() and torch.isfinite(back[[0, 1, 4]]).all() and (back[1] == 0).all() and scale[1] == 0
    assert torch.isnan(y[2]).all()
    # a whole row of the smallest weights: no scale that 32 bits hold
    codes, scale, _ = fb.fewbit_add_rms_norm_fwd(x[:1], weight=torch.full((40,), 1e-40, device="cuda"), bits=8)
    assert scale[0] == 0 and (codes.float() == 0).all()


@pytest.mark.gpu
def test_norm_past_32_bits_of_elements():
    rows, width = (1 << 20) + 5, 4096
    x = torch.zeros(rows, width, dtype=torch.bfloat16, device="cuda")
    x[-4:] = new((4, width), torch.bfloat16, 1)
    y, h = fb.fewbit_add_rms_norm_fwd(x, p=0.25, seed=3, place=1)
    mask = kept((4, width), 0.25, 3, 1, (rows - 4) * width).cuda()
    want = torch.where(mask, x[-4:].double() / 0.75, 0.0)
    assert ((h[-4:].double() - want).abs() <= 2.0 ** -7 * want.abs()).all() and torch.equal(h[-4:] != 0, mask & (x[-4:] != 0))
    del y
    g = x
    g[-4:] = new((4, width), torch.bfloat16, 2)
    gx, _, _ = fb.fewbit_add_rms_norm_bwd(g, None, h, p=0.25, seed=3, place=1, residual_grad=False, weight_grad=False)
    assert ((gx[-4:] != 0) <= mask).all() and (gx[-4:] != 0).double().mean() > 0.7


@pytest.mark.gpu
def test_the_counters_upper_half():
    """From element 2^34 on the generator's second counter counts; one row has elements on both sides."""
    width = 16376
    first_row = (1 << 34) // width
    rows = first_row + 3
    x = torch.ones(rows, width, dtype=torch.bfloat16, device="cuda")
    assert (1 << 34) % width and x.numel() > 1 << 34
    gx, _, _ = fb.fewbit_add_rms_norm_bwd(x, x, x, eps=0.0, p=0.25, seed=77, place=2, residual_grad=False, weight_grad=False)
    at = first_row * width // 4 * 4
    want = kept((3 * width,), 0.25, 77, 2, at).cuda()
    assert torch.equal(gx.view(-1)[at:at + 3 * width] != 0, want)
    del gx
    y = fb.fewbit_dropout_fwd(x, 0.25, seed=77, place=2, out=x)
    assert torch.equal(y.view(-1)[at:at + 3 * width] != 0, want)


@pytest.mark.gpu
def test_captured_graphs_draw_anew_and_streams_are_taken():
    x, r, g = (new((64, 512), torch.bfloat16, i) for i in range(3))
    seed = torch.zeros((), dtype=torch.int64, device="cuda")
    w = torch.ones(512, device="cuda")

    def step():
        y = fb.fewbit_dropout_fwd(x, 0.3, seed=seed, place=4)
        n, h = fb.fewbit_add_rms_norm_fwd(x, r, w, p=0.3, seed=seed, place=5)
        return (y, fb.fewbit_dropout_bwd(g, 0.3, seed=seed, place=4), n, h, *fb.fewbit_add_rms_norm_bwd(g, r, h, w, p=0.3, seed=seed, place=5))

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step()
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        held = step()
    for value in (5, -3, 1 << 40):
        seed.fill_(value)
        graph.replay()
        number = value % (1 << 64)
        want = (fb.fewbit_dropout_fwd(x, 0.3, seed=number, place=4), fb.fewbit_dropout_bwd(g, 0.3, seed=number, place=4))
        n, h = fb.fewbit_add_rms_norm_fwd(x, r, w, p=0.3, seed=number, place=5)
        want += (n, h, *fb.fewbit_add_rms_norm_bwd(g, r, h, w, p=0.3, seed=number, place=5))
        assert all(torch.equal(a, b) for a, b in zip(held, want))
    with torch.cuda.device(x.device):
        y = fb.fewbit_dropout_fwd(x, 0.3, seed=9, stream=side)
        n, h = fb.fewbit_add_rms_norm_fwd(x, r, w, stream=side)
        side.synchronize()
    assert torch.equal(y, fb.fewbit_dropout_fwd(x, 0.3, seed=9)) and torch.equal(n, fb.fewbit_add_rms_norm_fwd(x, r, w)[0])


@pytest.mark.gpu
def test_refusals_of_the_python_entry_points():
    x = new((4, 64), torch.float32, 0)
    for p in (-0.5, 1.0, float("nan")):
        with pytest.raises(ValueError, match="p must be"):
            fb.fewbit_dropout_fwd(x, p, seed=1)
    for call in (lambda: fb.fewbit_dropout_fwd(x.T, 0.1, seed=1), lambda: fb.fewbit_dropout_fwd(x.cpu(), 0.1, seed=1),
                 lambda: fb.fewbit_dropout_fwd(x.double(), 0.1, seed=1), lambda: fb.fewbit_dropout_fwd(x, 0.1, seed=1, place=-1),
                 lambda: fb.fewbit_dropout_fwd(x, 0.1, seed=1, residual=x[:2]), lambda: fb.fewbit_dropout_fwd(x, 0.1, seed=1, residual=x.bfloat16()),
                 lambda: fb.fewbit_dropout_fwd(x, 0.1, seed=torch.zeros(1, device="cuda")), lambda: fb.fewbit_dropout_fwd(x, 0.1, seed=torch.zeros(1, dtype=torch.int64)),
                 lambda: fb.fewbit_dropout_fwd(x, 0.1, seed=1, out=torch.empty(4, 64, device="cuda", dtype=torch.float16)),
                 lambda: fb.fewbit_dropout_fwd(x.view(-1)[:100], 0.1, seed=1, out=x.view(-1)[8:108]),
                 lambda: fb.fewbit_add_rms_norm_fwd(x.T), lambda: fb.fewbit_add_rms_norm_fwd(x, x[:2]), lambda: fb.fewbit_add_rms_norm_fwd(x, weight=torch.ones(63, device="cuda")),
                 lambda: fb.fewbit_add_rms_norm_fwd(x, weight=torch.ones(64, device="cuda").half()), lambda: fb.fewbit_add_rms_norm_fwd(x, bits=4),
                 lambda: fb.fewbit_add_rms_norm_bwd(x, None, x[:2]), lambda: fb.fewbit_add_rms_norm_bwd(x, x[:2], x), lambda: fb.fewbit_add_rms_norm_bwd(x.T, None, x.T)):
        with pytest.raises(ValueError):
            call()
    with pytest.raises(fb.FewbitError):
        fb.fewbit_add_rms_norm_fwd(torch.zeros(1, 16385, device="cuda"))
    with pytest.raises(fb.FewbitError):
        fb.fewbit_add_rms_norm_fwd(x, eps=-1.0)


@pytest.mark.gpu
def test_gradients_through_autograd():
    """Against the 64-bit formulas' own gradients, with the same mask: binary32, so 2^-16 of the size of the terms (at most 4)."""
    x, r = (new((6, 96), torch.float32, i).requires_grad_() for i in range(2))
    w = torch.rand(96, device="cuda", dtype=torch.bfloat16).requires_grad_()
    mask = kept((6, 96), 0.2, 31, 2).cuda()
    a, b, c = (new((6, 96), torch.float32, i) for i in (7, 8, 9))
    y, h = fb.fewbit_add_rms_norm(x, r, w, p=0.2, seed=31, place=2)
    z = fb.fewbit_dropout(h, 0.2, seed=31, place=2, residual=y)
    ((y * a).sum() + (h * b).sum() + (z * c).sum()).backward()
    x64, r64, w64 = (t.detach().double().requires_grad_() for t in (x, r, w))
    h64, y64, _, _ = norm_reference(x64, r64, w64, 1e-6, 0.2, mask)
    z64 = torch.where(mask, h64 / 0.8, 0.0) + y64
    ((y64 * a).sum() + (h64 * b).sum() + (z64 * c).sum()).backward()
    for t, t64 in ((x, x64), (r, r64)):
        assert ((t.grad.double() - t64.grad).abs() <= 2.0 ** -14).all()
    assert w.grad.dtype == torch.bfloat16 and ((w.grad.double() - w64.grad).abs() <= 2.0 ** -8 * w64.grad.abs() + 2.0 ** -14).all()

    # each of them alone, views and a type of its own, and no gradient of y or of h
    for used in (0, 1):
        xs = new((2, 3, 40), torch.bfloat16, 5).transpose(0, 1).requires_grad_()
        out = fb.fewbit_add_rms_norm(xs, None, None)
        out[used].float().sum().backward()
        assert xs.grad.shape == xs.shape and torch.isfinite(xs.grad).all()
        if used == 1:
            assert (xs.grad == 1).all()
    y0 = fb.fewbit_dropout(x, 0.0, seed=0)
    assert torch.equal(y0, x)
    # without residual and dropout h is x itself: both ways back to it, and an in-place change of it before the backward pass is seen
    xs = new((5, 40), torch.float32, 6).requires_grad_()
    y, h = fb.fewbit_add_rms_norm(xs, None, None)
    (y.sum() + 3 * h.sum()).backward()
    wide = xs.detach().double().requires_grad_()
    (norm_reference(wide, None, None, 1e-6, 0.0, torch.ones(5, 40, dtype=torch.bool, device="cuda"))[1].sum() + 3 * wide.sum()).backward()
    assert ((xs.grad.double() - wide.grad).abs() <= 2.0 ** -14).all()
    y, _ = fb.fewbit_add_rms_norm(xs, None, None)
    with torch.no_grad():
        xs.add_(1)
    with pytest.raises(RuntimeError, match="modified by an inplace operation"):
        y.sum().backward()


@pytest.mark.gpu
def test_a_seed_changed_before_the_backward_pass_is_an_error_and_second_derivatives_are_refused():
    seed = torch.tensor(3, device="cuda")
    x = new((4, 64), torch.float32, 0).requires_grad_()
    for call in (lambda: fb.fewbit_dropout(x, 0.5, seed=seed), lambda: fb.fewbit_add_rms_norm(x, None, None, p=0.5, seed=seed)[0]):
        out = call()
        seed.add_(1)
        with pytest.raises(RuntimeError, match="modified by an inplace operation"):
            out.sum().backward()
        (dx,) = torch.autograd.grad(call().square().sum(), x, create_graph=True)
        with pytest.raises(RuntimeError, match="once_differentiable"):
            dx.sum().backward()


@pytest.mark.gpu
def test_gradients_against_differences():
    """Central differences of the 32-bit forward pass itself: step 2^-6, curvature and rounding leave 2^-7 of gradients of size 1."""
    x, r = new((2, 24), torch.float32, 1), new((2, 24), torch.float32, 2)
    w, a = new((24,), torch.float32, 3), new((2, 24), torch.float32, 4)
    kw = {"p": 0.25, "seed": 8, "place": 1}

    def value(xx, rr, ww):
        y, h = fb.fewbit_add_rms_norm_fwd(xx, rr, ww, **kw)
        return ((y.double() + h.double()) * a.double()).sum()

    _, h = fb.fewbit_add_rms_norm_fwd(x, r, w, **kw)
    grads = fb.fewbit_add_rms_norm_bwd(a, a, h, w, **kw)
    for which, t in enumerate((x, r, w)):
        for i in range(0, t.numel(), 5):
            step = torch.zeros_like(t).view(-1)
            step[i] = 2.0 ** -6
            step = step.view_as(t)
            args = [x, r, w]
            args[which] = t + step
            up = value(*args)
            args[which] = t - step
            slope = (up - value(*args)) * 32
            assert abs(float(slope) - float(grads[which].view(-1)[i])) <= 2.0 ** -7 * max(1.0, abs(float(slope)))
