"""A small encoder trained with the operators around attention's scores and the residual stream: a learned bias of relative
positions by buckets that all layers share, documents packed into one row that do not see each other, branches that go through
dropout into the residual stream and its norm in one pass, GELU that keeps 3 bits an element, AdamW with 8-bit moments.  The task
is synthetic: every token is to be told from its two neighbours' sum.

    python examples/train_encoder.py [--steps 200] [--width 256] [--layers 2] [--length 256]
"""
import argparse
import os
import sys

import torch
from torch import nn

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
import paper_2202_00441_b200 as fb  # noqa: E402


class Layer(nn.Module):
    """Takes a branch and the residual stream, returns the next branch and the stream."""

    def __init__(self, width: int, heads: int, p: float, place: int):
        super().__init__()
        self.heads, self.p, self.place = heads, p, place
        self.norm1, self.norm2 = nn.Parameter(torch.ones(width)), nn.Parameter(torch.ones(width))
        self.qkv, self.out = nn.Linear(width, 3 * width, bias=False), nn.Linear(width, width, bias=False)
        self.up, self.up_bias = nn.Linear(width, 4 * width, bias=False), nn.Parameter(torch.zeros(4 * width))
        self.act, self.down = fb.FewBitActivation("gelu", bits=3), nn.Linear(4 * width, width)

    def forward(self, branch, stream, bias, documents, seed):
        p = self.p if self.training else 0.0
        x, stream = fb.fewbit_add_rms_norm(branch, stream, self.norm1, p=p, seed=seed, place=2 * self.place)
        b, n, width = x.shape
        q, k, v = self.qkv(x).view(b, n, 3, self.heads, width // self.heads).unbind(2)
        a = fb.fewbit_attention(q, k, v, distance_bias=bias, q_documents=documents, k_documents=documents, cap=30.0)
        x, stream = fb.fewbit_add_rms_norm(self.out(a.reshape(b, n, width)), stream, self.norm2, p=p, seed=seed, place=2 * self.place + 1)
        return self.down(self.act(self.up(x), self.up_bias)), stream


class Model(nn.Module):
    def __init__(self, vocab: int = 32, width: int = 256, layers: int = 2, heads: int = 4, p: float = 0.1, buckets: int = 32, reach: int = 64):
        super().__init__()
        self.embed = nn.Embedding(vocab, width)
        self.layers = nn.ModuleList(Layer(width, heads, p, i) for i in range(layers))
        self.bias, self.reach, self.p = nn.Parameter(torch.zeros(buckets, heads)), reach, p
        self.norm, self.head = nn.RMSNorm(width), nn.Linear(width, vocab, bias=False)

    def forward(self, tokens, documents, seed: int = 0):
        bias = fb.fewbit_relative_bias(self.bias, self.reach, bidirectional=True)
        branch, stream = self.embed(tokens), None
        for layer in self.layers:
            branch, stream = layer(branch, stream, bias, documents, seed)
        stream = fb.fewbit_dropout(branch, self.p if self.training else 0.0, seed=seed, place=1 << 20, residual=stream)
        return self.head(self.norm(stream))


def batch(gen, size: int, length: int, vocab: int):
    """Tokens, their documents (runs of random length) and what is asked: the sum of both neighbours in the document."""
    tokens = torch.randint(0, vocab, (size, length), generator=gen, device="cuda")
    documents = (torch.rand(size, length, generator=gen, device="cuda") < 8 / length).int().cumsum(1, dtype=torch.int32)
    same = documents[:, 1:] == documents[:, :-1]
    answer = torch.zeros_like(tokens)
    answer[:, 1:] += torch.where(same, tokens[:, :-1], 0)
    answer[:, :-1] += torch.where(same, tokens[:, 1:], 0)
    return tokens, documents, answer % vocab


def train(steps: int = 200, width: int = 256, layers: int = 2, length: int = 256, size: int = 16, vocab: int = 32, seed: int = 0, log=None):
    """Returns the losses of all steps and the model."""
    torch.manual_seed(seed)
    model = Model(vocab, width, layers).cuda().bfloat16()
    optimizer = fb.FewBitAdamW(model.parameters(), lr=2e-3, weight_decay=0.01, seed=seed)
    gen = torch.Generator(device="cuda").manual_seed(seed)
    losses = []
    for step in range(steps):
        tokens, documents, answer = batch(gen, size, length, vocab)
        loss = nn.functional.cross_entropy(model(tokens, documents, seed=seed * steps + step).float().flatten(0, 1), answer.flatten())
        loss.backward()
        optimizer.step()
        if step + 1 < steps:
            optimizer.zero_grad(set_to_none=True)
        losses.append(loss.detach())
        if log and (step % 50 == 0 or step == steps - 1):
            log(f"step {step:4d}  loss {float(losses[-1]):.4f}")
    return [float(x) for x in losses], model


if __name__ == "__main__":
    ap = argparse.ArgumentParser(description=__doc__, formatter_class=argparse.RawDescriptionHelpFormatter)
    for name, default in (("steps", 200), ("width", 256), ("layers", 2), ("length", 256)):
        ap.add_argument("--" + name, type=int, default=default)
    a = ap.parse_args()
    before = fb.fewbit_launch_count()
    train(a.steps, a.width, a.layers, a.length, log=print)
    print(f"{fb.fewbit_launch_count() - before} kernels of the library, {torch.cuda.max_memory_allocated() / 2 ** 20:.0f} MiB at most")
