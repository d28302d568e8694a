"""The residual stream's operators where they can go wrong beside the formulas' ordinary values; tolerances as in test_residual.py."""
import pytest
import torch

import paper_2202_00441_b200 as fb
import test_residual as tr

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", tr.TYPES, ids=str)
@pytest.mark.parametrize("rows,width,offset", [(5, 256, 0), (1, 64, 0), (7, 333, 0), (3, 20, 0), (1000, 509, 0), (2, 100, 1), (5, 640, 0), (3, 2052, 0), (2999, 128, 0)])
def test_weight_gradients_without_eps(rows, width, offset, dtype):
    """eps = 0 and rows that leave some of a CTA's places without one: what such a place adds to the sums is 0."""
    gy, h, w = tr.new((rows, width), dtype, 1, 1.0, offset), tr.new((rows, width), dtype, 2, 2.0, offset), tr.new((width,), torch.float32, 3, 0.3) + 1
    gx, _, gw = fb.fewbit_add_rms_norm_bwd(gy, None, h, w, eps=0.0)
    hd, gd = h.double(), gy.double()
    s = hd.square().mean(-1, keepdim=True).rsqrt()
    terms = gd * hd * s
    assert ((gw.double() - terms.sum(0)).abs() <= ((rows + 40) * 2.0 ** -24 + 2.0 ** -18) * terms.abs().sum(0)).all()
    g, u = gd * w.double(), hd * s
    want = s * (g - u * (g * u).mean(-1, keepdim=True))
    bound = tr.E[dtype] * want.abs() + tr.TINY[dtype] + 2.0 ** -17 * (s * g.abs() + s * u.abs() * (g * u).abs().mean(-1, keepdim=True))
    assert ((gx.double() - want).abs() <= bound).all()


@pytest.mark.parametrize("p", [0.0, 0.3])
def test_a_gradient_that_reaches_the_stream_alone(p):
    """Where the normed result is not used, the norm has no part in the gradient: rows whose norm is not finite do not touch it, and the
    weight has none."""
    x, r, g = (tr.new((6, 96), torch.float32, i) for i in range(3))
    r[1] = float("inf")
    r[2] = float("nan")
    x[3] = r[3] = 0
    x, r = x.requires_grad_(), r.requires_grad_()
    w = torch.ones(96, device="cuda").requires_grad_()
    before = fb.fewbit_launch_count()
    _, h = fb.fewbit_add_rms_norm(x, r, w, eps=0.0, p=p, seed=8, place=3)
    h.backward(g)
    assert fb.fewbit_launch_count() - before == (2 if p else 1)
    assert torch.equal(r.grad, g) and w.grad is None
    assert torch.equal(x.grad, fb.fewbit_dropout_bwd(g, p, seed=8, place=3) if p else g)
    seed = torch.tensor(8, device="cuda")
    _, h = fb.fewbit_add_rms_norm(x, None, w, eps=0.0, p=p, seed=seed, place=3)
    (gx,) = torch.autograd.grad(h, x, g)
    assert torch.equal(gx, x.grad)


def test_probabilities_next_to_one():
    """From 1 - 2^-33 on round(p 2^32) is above every word: nothing is kept, not even the largest, which element 1 has with this seed."""
    seed, x = 454088803, torch.ones(64, device="cuda")
    for p, kept in ((1 - 2.0 ** -32, 2.0 ** 32), (1 - 2.0 ** -40, 0.0), (1 - 2.0 ** -53, 0.0)):
        for y in (fb.fewbit_dropout_fwd(x, p, seed=seed), fb.fewbit_dropout_bwd(x, p, seed=seed), fb.fewbit_add_rms_norm_fwd(x[None], p=p, seed=seed)[1][0]):
            assert y[1] == kept and (y[:1] == 0).all() and (y[2:] == 0).all()
