"""What the operators' Python entry points refuse before anything is launched or kept."""
import types

import pytest
import torch

import paper_2202_00441_b200 as fb
import test_qk_norm_rope as tq
from paper_2202_00441_b200 import operators as ops


def test_a_stream_of_another_device_is_refused():
    """Stand-ins: the check needs devices only, and no second GPU."""
    recorded = []

    def tensor(index):
        return types.SimpleNamespace(device=torch.device("cuda", index), record_stream=lambda s: recorded.append(index))

    stream = types.SimpleNamespace(device=torch.device("cuda", 1))
    for tensors in ((tensor(0),), (tensor(1), None, tensor(0))):
        with pytest.raises(ValueError, match="device"):
            ops._On(stream, *tensors)
    assert recorded == []


@pytest.mark.gpu
def test_outputs_that_overlap_are_refused():
    """Elements that share memory with one another, or with other elements of an input, would be written in any order."""
    flat = torch.randn(2, 3 * 5 * 4 * 64 + 64, device="cuda")
    n = 3 * 5 * 4 * 64
    q, k = (x[:n].view(3, 5, 4, 64) for x in flat)
    moved_q, moved_k = (x[64:64 + n].view(3, 5, 4, 64) for x in flat)
    same = torch.empty(1, 1, 1, 64, device="cuda").expand(3, 5, 4, 64)
    c, s = tq.tables(5, 64)
    new = torch.empty_like(q)
    g = torch.randn_like(q)
    for out in ((same, new), (new, same), (moved_q, new), (new, moved_k), (k, new), (new, q), (new, new)):
        with pytest.raises(ValueError, match="overlap"):
            fb.fewbit_qk_norm_rope_fwd(q, k, None, None, c, s, out=out)
        with pytest.raises(ValueError, match="overlap"):
            fb.fewbit_qk_norm_rope_bwd(g, g.clone(), q, k, None, None, c, s, out=out, weight_grads=False)
    with pytest.raises(ValueError, match="overlap"):
        fb.fewbit_qk_norm_rope_bwd(moved_q.contiguous(), moved_k, q, k.clone(), None, None, c, s, out=(new, k), weight_grads=False)
    want = fb.fewbit_qk_norm_rope_fwd(q, k, None, None, c, s)
    fb.fewbit_qk_norm_rope_fwd(q, k, None, None, c, s, out=(q, k))
    assert torch.equal(q, want[0]) and torch.equal(k, want[1])


@pytest.mark.gpu
def test_sizes_past_31_bits_are_refused():
    x = torch.zeros(1, 1, 1, 8, device="cuda", dtype=torch.bfloat16)
    many = 2 ** 32 + 1
    for shape in ((many, 1, 1, 8), (1, 1, many, 8)):
        big = x.expand(shape)
        with pytest.raises(ValueError, match="too large"):
            fb.fewbit_attention_fwd(big, big, big)
        with pytest.raises(ValueError, match="too large"):
            fb.fewbit_qk_norm_rope_fwd(big, big, None, None, None, None)


@pytest.mark.gpu
def test_a_refused_parameter_group_is_not_kept():
    p = torch.nn.Parameter(torch.zeros(8, device="cuda"))
    opt = fb.FewBitAdamW([p])
    with pytest.raises(ValueError):
        opt.add_param_group({"params": [torch.nn.Parameter(torch.zeros(4))]})
    assert len(opt.param_groups) == 1
    p.grad = torch.ones_like(p)
    opt.step()
