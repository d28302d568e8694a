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
