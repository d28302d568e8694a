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
