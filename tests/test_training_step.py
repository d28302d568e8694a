"""The operators as a training program uses them: gradients through autograd against a plain 64-bit model of the same
formulas, the optimizer against its formula and through a checkpoint, and the example, which runs them all together."""
import copy
import io
import os
import sys

import pytest
import torch

import paper_2202_00441_b200 as fb
import test_attention as ta
import test_qk_norm_rope as tq

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
pytestmark = pytest.mark.gpu


def test_attention_gradients_reach_views_of_one_projection():
    """q, k, v as slices of one tensor, once transposed so that the library does not take the strides as they are."""
    for transpose in (False, True):
        torch.manual_seed(0)
        x = torch.randn(2, 70, 8, 64, device="cuda").bfloat16()
        if transpose:
            x = x.transpose(1, 3).contiguous().transpose(1, 3)
        x.requires_grad_()
        out = fb.fewbit_attention(x[:, :, :4], x[:, :, 4:6], x[:, :, 6:], causal=True)
        g = torch.randn(out.shape, device="cuda").bfloat16()
        out.backward(g)
        d = x.detach()
        for i in range(2):
            got = {"out": out[i], "lse": fb.fewbit_attention_fwd(d[:, :, :4].contiguous(), d[:, :, 4:6].contiguous(), d[:, :, 6:].contiguous(), causal=True)[1][i],
                   "dq": x.grad[i, :, :4], "dk": x.grad[i, :, 4:6], "dv": x.grad[i, :, 6:]}
            ta.compare(d[i, :, :4], d[i, :, 4:6], d[i, :, 6:], g[i], {k: v.detach() for k, v in got.items()}, True, 64 ** -0.5)


def test_an_expanded_input_and_an_expanded_gradient():
    """Keys and values broadcast over the batch: their gradients are the sums over it (each rounded to bfloat16, then added by
    autograd in bfloat16: 3 terms, 3 roundings of at most 2^-8 of the sum of magnitudes).  A gradient that is one number expanded."""
    torch.manual_seed(1)
    q = torch.randn(3, 40, 2, 64, device="cuda").bfloat16()
    kv = torch.randn(1, 33, 2, 64, device="cuda").bfloat16().requires_grad_()
    out = fb.fewbit_attention(q, kv.expand(3, -1, -1, -1), kv.expand(3, -1, -1, -1))
    out.sum().backward()
    total, size = 0, 0
    for i in range(3):
        g = torch.ones(40, 2, 64, dtype=torch.float64, device="cuda")
        r, _ = ta.reference(q[i].double(), kv[0].detach().double(), kv[0].detach().double(), g, False, 64 ** -0.5)
        total, size = total + r["dk"] + r["dv"], size + r["dk"].abs() + r["dv"].abs()
    err = (kv.grad[0].double() - total.transpose(0, 1)).abs()
    assert (err <= 8 * 2.0 ** -8 * size.transpose(0, 1) + 0.05).all()


def test_head_norm_gradients_and_weight_types():
    q, k, _, c, s, p = tq.inputs(2, 9, 4, 2, 64, 64, torch.float32, "fused", torch.int64, True)
    q, k = q.clone().requires_grad_(), k.clone().requires_grad_()
    w = [torch.rand(64, device="cuda", dtype=torch.bfloat16, requires_grad=True) for _ in range(2)]
    a, b = fb.fewbit_qk_norm_rope(q, k, *w, c, s, positions=p)
    (a.square().sum() + b.sum()).backward()
    cc, ss = tq.gathered(c, s, p, 2, 9, 64)
    for x, wt, loss in ((q, w[0], lambda y: y.square().sum()), (k, w[1], lambda y: y.sum())):
        x64, w64 = x.detach().double().requires_grad_(), wt.detach().double().requires_grad_()
        loss(tq.forward(x64, w64, cc, ss, 1e-6, False)).backward()
        assert torch.allclose(x.grad.double(), x64.grad, rtol=1e-4, atol=1e-4)        # 32-bit sums of 64 terms, gradients of size 1
        assert wt.grad.dtype == torch.bfloat16
        assert ((wt.grad.double() - w64.grad).abs() <= 2.0 ** -8 * w64.grad.abs() + 1e-3).all()


def parameters(seed=0, dtype=torch.bfloat16):
    g = torch.Generator(device="cuda").manual_seed(seed)
    return [torch.nn.Parameter((torch.randn(n, generator=g, device="cuda") * 0.1).to(dtype)) for n in (1000, 300, 7)]


def set_grads(params, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    for p in params:
        p.grad = (torch.randn(p.shape, generator=g, device="cuda") * 0.01).to(p.dtype)


def test_optimizer_with_32_bit_moments_follows_the_formula():
    params = parameters(dtype=torch.float32)
    opt = fb.FewBitAdamW(params, lr=1e-2, state_bits=32, weight_decay=0.1)
    ref = [(p.detach().double(), torch.zeros_like(p, dtype=torch.float64), torch.zeros_like(p, dtype=torch.float64)) for p in params]
    for step in range(1, 6):
        set_grads(params, step)
        opt.step()
        for i, p in enumerate(params):
            x, m, v = ref[i]
            g = p.grad.double()
            m, v = 0.9 * m + 0.1 * g, 0.999 * v + 0.001 * g * g
            x = x * (1 - 1e-3) - 1e-2 * (m / (1 - 0.9 ** step)) / ((v / (1 - 0.999 ** step)).sqrt() + 1e-8)
            ref[i] = (x, m, v)
            assert ((p.double() - x).abs() <= 5 * 2.0 ** -20 * (x.abs() + 1e-2)).all()   # 5 steps of some 16 roundings each


def test_optimizer_groups_missing_gradients_and_checkpoint():
    def run(restart):
        params = parameters()
        opt = fb.FewBitAdamW([{"params": params[:2]}, {"params": params[2:], "lr": 1e-2, "state_bits": 32}], lr=3e-3, seed=5)
        for step in range(6):
            set_grads(params, step)
            if step == 2:
                params[1].grad = None                        # this one falls a step behind
            opt.step(grad_scale=torch.tensor(0.5, device="cuda"))
            if restart and step == 3:
                buf = io.BytesIO()
                torch.save((opt.state_dict(), [p.detach() for p in params]), buf)
                buf.seek(0)
                state, values = torch.load(buf, weights_only=True)
                params = [torch.nn.Parameter(v.clone()) for v in values]
                opt = fb.FewBitAdamW([{"params": params[:2]}, {"params": params[2:], "lr": 1e-2, "state_bits": 32}], lr=3e-3, seed=5)
                opt.load_state_dict(state)
                assert opt.state[params[0]]["exp_avg"].dtype == torch.float8_e4m3fn and opt.state[params[0]]["master"].dtype == torch.float32
        return params, opt

    a, opt = run(False)
    b, _ = run(True)
    assert all(torch.equal(x, y) for x, y in zip(a, b))
    assert [opt.state[p]["step"] for p in a] == [6, 5, 6]
    c = copy.deepcopy(opt)
    set_grads([p for g in c.param_groups for p in g["params"]], 9)
    c.step()


def test_optimizer_refuses():
    p = parameters()
    with pytest.raises(ValueError):
        fb.FewBitAdamW(p, state_bits=4)
    with pytest.raises(ValueError):
        fb.FewBitAdamW([torch.nn.Parameter(torch.zeros(4))])
    with pytest.raises(ValueError):
        fb.FewBitAdamW([torch.nn.Parameter(torch.zeros(4, 6, device="cuda").t())])


def test_example_learns():
    sys.path.insert(0, os.path.join(ROOT, "examples"))
    import train_block
    losses = train_block.train(steps=300)
    assert losses[0] > 3.5                                   # log(64) = 4.16: nothing known
    assert sum(losses[-10:]) / 10 < 0.5                      # the repetition is found
    assert fb.fewbit_attention_timeout_count() == 0
