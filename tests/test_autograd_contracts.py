"""What autograd promises beyond the gradients' values: what the backward pass reads has not been changed since, and what has no
gradient says so."""
import pytest
import torch

import paper_2202_00441_b200 as fb
import test_qk_norm_rope as tq


def _packed():
    x = torch.randn(40, 4, 64, device="cuda").bfloat16()
    q, k, v = (t.clone().requires_grad_() for t in (x[:, :2], x[:, 2:3], x[:, 3:]))
    return q, k, v, torch.tensor([0, 15, 40], dtype=torch.int32, device="cuda"), torch.tensor([0, 15, 40], dtype=torch.int32, device="cuda")


@pytest.mark.gpu
@pytest.mark.parametrize("which", [0, 1])
def test_offsets_changed_before_the_backward_pass_are_an_error(which):
    q, k, v, *offsets = _packed()
    out = fb.fewbit_attention(q, k, v, causal=True, q_offsets=offsets[0], k_offsets=offsets[1], max_q_len=40, max_k_len=40)
    offsets[which].copy_(torch.tensor([0, 30, 40]))              # the next micro-batch's, in the same buffer
    with pytest.raises(RuntimeError, match="modified by an inplace operation"):
        out.sum().backward()


@pytest.mark.gpu
@pytest.mark.parametrize("which", ["cos", "sin", "positions"])
def test_tables_and_positions_changed_before_the_backward_pass_are_an_error(which):
    q, k, w, c, s, p = tq.inputs(1, 9, 2, 1, 64, 64, torch.float32, "fused", torch.int32, True)
    q, k = q.clone().requires_grad_(), k.clone().requires_grad_()
    a, b = fb.fewbit_qk_norm_rope(q, k, *w, c, s, positions=p)
    {"cos": c, "sin": s, "positions": p}[which].zero_()
    with pytest.raises(RuntimeError, match="modified by an inplace operation"):
        (a.sum() + b.sum()).backward()


@pytest.mark.gpu
def test_tables_that_want_a_gradient_are_refused():
    q, k, w, c, s, _ = tq.inputs(1, 9, 2, 1, 64, 64, torch.float32, "fused", None, True)
    for cos, sin in ((c.clone().requires_grad_(), s), (c, s.clone().requires_grad_())):
        with pytest.raises(ValueError, match="cos and sin"):
            fb.fewbit_qk_norm_rope(q, k, *w, cos, sin)
        with torch.no_grad():
            fb.fewbit_qk_norm_rope(q, k, *w, cos, sin)


@pytest.mark.gpu
def test_second_derivatives_are_refused():
    q, k, v, *offsets = _packed()
    out = fb.fewbit_attention(q, k, v, q_offsets=offsets[0], k_offsets=offsets[1], max_q_len=40, max_k_len=40)
    (dq,) = torch.autograd.grad(out.float().square().sum(), q, create_graph=True)
    with pytest.raises(RuntimeError, match="once_differentiable"):
        dq.float().sum().backward()
    q, k, w, c, s, _ = tq.inputs(1, 9, 2, 1, 64, 64, torch.float32, "fused", None, True)
    q = q.clone().requires_grad_()
    a, b = fb.fewbit_qk_norm_rope(q, k, *w, c, s)
    (dq,) = torch.autograd.grad(a.square().sum() + b.sum(), q, create_graph=True)
    with pytest.raises(RuntimeError, match="once_differentiable"):
        dq.sum().backward()
