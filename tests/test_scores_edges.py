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
