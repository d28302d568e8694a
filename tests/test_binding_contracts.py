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
