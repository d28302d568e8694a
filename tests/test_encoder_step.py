"""The operators around attention's scores and the residual stream as a training program runs them together: a chain of norm,
attention with a learned bias, cap, prefix and documents, dropout and norm against the same chain in 64 bits with the same masks; the
example, which runs them with the few-bit activation and the optimizer; what a captured step gives."""
import os
import sys

import pytest
import torch

import paper_2202_00441_b200 as fb
import test_attention_scores as ts
import test_residual as tr

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
pytestmark = pytest.mark.gpu
B, N, H, HK, D, W = 2, 150, 4, 2, 32, 128


def inputs(dtype):
    gen = torch.Generator(device="cuda").manual_seed(5)

    def new(*shape, size=1.0, to=dtype):
        return (torch.randn(*shape, generator=gen, device="cuda") * size).to(to).requires_grad_()

    leaves = {"branch": new(B, N, W), "stream": new(B, N, W), "w1": new(W, size=0.3, to=torch.float32), "w2": new(W, size=0.3, to=torch.float32),
              "table": new(16, H, to=torch.float32), "qkv": new(W, (H + 2 * HK) * D, size=W ** -0.5), "out": new(H * D, W, size=(H * D) ** -0.5)}
    docs = torch.randint(0, 3, (B, N), generator=gen, device="cuda", dtype=torch.int32).sort(1).values
    prefix = torch.tensor([40, 0], dtype=torch.int32, device="cuda")
    return leaves, docs, prefix


def chain(x, docs, prefix, seed):
    h1, s1 = fb.fewbit_add_rms_norm(x["branch"], x["stream"], x["w1"], p=0.2, seed=seed, place=0)
    y = (h1.view(-1, W) @ x["qkv"]).view(B, N, H + 2 * HK, D)
    bias = fb.fewbit_relative_bias(x["table"], 20)
    a = fb.fewbit_attention(y[:, :, :H], y[:, :, H:H + HK], y[:, :, H + HK:], causal=True, distance_bias=bias, cap=4.0, prefix_lens=prefix, q_documents=docs, k_documents=docs)
    branch = (a.reshape(-1, H * D) @ x["out"]).view(B, N, W)
    h2, s2 = fb.fewbit_add_rms_norm(branch, s1, x["w2"], p=0.1, seed=seed, place=1)
    return fb.fewbit_dropout(h2, 0.3, seed=seed, place=2, residual=s2)


def plain_chain(x, docs, prefix, seed):
    mask = [tr.kept((B, N, W), p, seed, place).cuda() for p, place in ((0.2, 0), (0.1, 1), (0.3, 2))]
    flat = lambda t: t.view(-1, W)  # noqa: E731
    s1, h1, _, _ = tr.norm_reference(flat(x["branch"]), flat(x["stream"]), x["w1"], 1e-6, 0.2, flat(mask[0]))
    y = (h1 @ x["qkv"]).view(B, N, H + 2 * HK, D)
    of = ts.exact_buckets(16, 20, False)
    bias = x["table"][of].T
    away = torch.arange(N, device="cuda")[None] - torch.arange(N, device="cuda")[:, None]
    q, k, v = (t.transpose(1, 2) for t in (y[:, :, :H], y[:, :, H:H + HK].repeat_interleave(H // HK, 2), y[:, :, H + HK:].repeat_interleave(H // HK, 2)))
    z = 4.0 * (q @ k.transpose(2, 3) * D ** -0.5 / 4.0).tanh() + bias[:, away.clamp(-20, 20) + 20]
    seen = ((away <= 0)[None] | (torch.arange(N, device="cuda")[None, None] < prefix[:, None, None])) & (docs[:, :, None] == docs[:, None, :])
    a = z.masked_fill(~seen[:, None], -torch.inf).softmax(-1) @ v
    s2, h2, _, _ = tr.norm_reference((a.transpose(1, 2).reshape(-1, H * D) @ x["out"]), s1, x["w2"], 1e-6, 0.1, flat(mask[1]))
    return (torch.where(flat(mask[2]), h2 / 0.7, 0.0) + s2).view(B, N, W)


def test_a_block_and_its_gradients():
    """binary16.  Twenty roundings of 2^-11 in a row, forward and backward, each of which moves the 2-norm of what follows by at most
    about as much: 2^-6 in all leaves room for a factor of 1.6."""
    leaves, docs, prefix = inputs(torch.float16)
    g = torch.randn(B, N, W, generator=torch.Generator(device="cuda").manual_seed(9), device="cuda").half()
    out = chain(leaves, docs, prefix, 1234)
    out.backward(g)
    wide = {k: v.detach().double().requires_grad_() for k, v in leaves.items()}
    want = plain_chain(wide, docs, prefix, 1234)
    want.backward(g.double())
    off = lambda a, b: float((a.double() - b).norm() / b.norm())  # noqa: E731
    assert off(out.detach(), want.detach()) <= 2.0 ** -6
    for name in leaves:
        assert leaves[name].grad.dtype == leaves[name].dtype and off(leaves[name].grad, wide[name].grad) <= 2.0 ** -6, name


def test_a_captured_step_follows_its_seed_and_masks():
    """Forward and backward captured once; replayed with another seed, other documents and prefixes in the same buffers it gives what
    eager calls give."""
    leaves, docs, prefix = inputs(torch.bfloat16)
    seed = torch.tensor(7, device="cuda")
    g = torch.ones(B, N, W, device="cuda", dtype=torch.bfloat16)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        torch.autograd.grad(chain(leaves, docs, prefix, seed), list(leaves.values()), g)
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = chain(leaves, docs, prefix, seed)
        grads = torch.autograd.grad(out, list(leaves.values()), g)
    for i in range(3):
        seed.fill_(100 + i)
        docs.copy_(torch.randint(0, 4, docs.shape, device="cuda", dtype=torch.int32).sort(1).values)
        prefix.fill_(30 * i)
        graph.replay()
        again = chain(leaves, docs, prefix, 100 + i)
        want = torch.autograd.grad(again, list(leaves.values()), g)
        assert torch.equal(out, again) and all(torch.equal(a, b) for a, b in zip(grads, want))


def test_two_streams_at_once():
    """The same block on two streams, started together, many times: each gives what it gives alone."""
    leaves, docs, prefix = inputs(torch.bfloat16)
    g = torch.ones(B, N, W, device="cuda", dtype=torch.bfloat16)

    def step(seed):
        out = chain(leaves, docs, prefix, seed)
        return (out, *torch.autograd.grad(out, list(leaves.values()), g))

    alone = [step(s) for s in (1, 2)]
    streams = [torch.cuda.Stream() for _ in range(2)]
    torch.cuda.synchronize()
    got = [[], []]
    for _ in range(5):
        for i, s in enumerate(streams):
            with torch.cuda.stream(s):
                got[i].append(step(i + 1))
    torch.cuda.synchronize()
    for i in range(2):
        for one in got[i]:
            assert all(torch.equal(a, b) for a, b in zip(one, alone[i]))


def test_the_example_runs():
    sys.path.insert(0, os.path.join(ROOT, "examples"))
    import train_encoder

    before = fb.fewbit_launch_count()
    losses, model = train_encoder.train(steps=3, width=128, layers=2, length=96, size=4)
    assert len(losses) == 3 and all(x == x and x < 100 for x in losses)
    assert all(p.grad is not None and torch.isfinite(p.grad).all() and (p.grad != 0).any() for p in model.parameters())
    assert fb.fewbit_launch_count() - before > 3 * 2 * 10
    model.eval()
    tokens, documents, _ = train_encoder.batch(torch.Generator(device="cuda").manual_seed(1), 2, 50, 32)
    with torch.no_grad():
        whole = model(tokens, documents)
        cut = int((documents[0] == documents[0, 0]).sum())       # the first document alone gives the same: the others are not seen
        alone = model(tokens[:1, :cut], documents[:1, :cut])
    assert (whole[0, :cut].float() - alone[0].float()).abs().max() <= 0.1 * whole.float().abs().max()
