"""A small causal transformer trained with everything that keeps little for the backward pass: attention whose
probabilities are recomputed, the head norm fused with the rotation, GELU that keeps 3 bits an element, AdamW with
8-bit moments.  The task is synthetic: the second half of each sequence repeats the first.

    python examples/train_block.py [--steps 300] [--width 256] [--layers 2] [--length 128]
"""
import argparse
import os
import sys

import torch
from torch import nn

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
import paper_2202_00441_b200 as fb  # noqa: E402


class Block(nn.Module):
    def __init__(self, width: int, heads: int, kv_heads: int, head_dim: int):
        super().__init__()
        self.heads, self.kv_heads, self.head_dim = heads, kv_heads, head_dim
        self.norm1, self.norm2 = nn.RMSNorm(width), nn.RMSNorm(width)
        self.qkv = nn.Linear(width, (heads + 2 * kv_heads) * head_dim, bias=False)
        self.q_weight, self.k_weight = nn.Parameter(torch.ones(head_dim)), nn.Parameter(torch.ones(head_dim))
        self.out = nn.Linear(heads * head_dim, width, bias=False)
        self.up, self.up_bias = nn.Linear(width, 4 * width, bias=False), nn.Parameter(torch.zeros(4 * width))
        self.act, self.down = fb.FewBitActivation("gelu", bits=3), nn.Linear(4 * width, width)

    def forward(self, x, cos, sin):
        b, n, _ = x.shape
        h, hk = self.heads, self.kv_heads
        qkv = self.qkv(self.norm1(x)).view(b, n, h + 2 * hk, self.head_dim)
        q, k = fb.fewbit_qk_norm_rope(qkv[:, :, :h], qkv[:, :, h:h + hk], self.q_weight, self.k_weight, cos, sin)
        a = fb.fewbit_attention(q, k, qkv[:, :, h + hk:], causal=True)
        x = x + self.out(a.reshape(b, n, -1))
        return x + self.down(self.act(self.up(self.norm2(x)), self.up_bias))


class Model(nn.Module):
    def __init__(self, vocab: int = 64, width: int = 256, layers: int = 2, heads: int = 4, kv_heads: int = 2, head_dim: int = 64,
                 length: int = 128):
        super().__init__()
        self.embed = nn.Embedding(vocab, width)
        self.blocks = nn.ModuleList(Block(width, heads, kv_heads, head_dim) for _ in range(layers))
        self.norm, self.head = nn.RMSNorm(width), nn.Linear(width, vocab, bias=False)
        angle = torch.arange(length)[:, None] * 1000.0 ** (-torch.arange(0, head_dim, 2) / head_dim)
        self.cos, self.sin = nn.Buffer(angle.cos()), nn.Buffer(angle.sin())

    def forward(self, tokens):
        x = self.embed(tokens)
        for block in self.blocks:
            x = block(x, self.cos, self.sin)
        return self.head(self.norm(x))


def batch(gen, size: int, length: int, vocab: int):
    half = torch.randint(0, vocab, (size, length // 2), generator=gen, device="cuda")
    return torch.cat([half, half], 1)


def loss_of(model, tokens):
    logits = model(tokens[:, :-1]).float()
    start = tokens.shape[1] // 2 - 1                                 # what can be known: the second half
    return nn.functional.cross_entropy(logits[:, start:].flatten(0, 1), tokens[:, start + 1:].flatten())


def train(steps: int = 300, width: int = 256, layers: int = 2, length: int = 128, size: int = 32, vocab: int = 64, seed: int = 0,
          state_bits: int = 8, log=None):
    """Returns the losses of all steps."""
    torch.manual_seed(seed)
    model = Model(vocab, width, layers, length=length).cuda()
    cos, sin = model.cos, model.sin
    model.bfloat16()
    model.cos, model.sin = cos, sin                                  # the tables stay in binary32
    optimizer = fb.FewBitAdamW(model.parameters(), lr=2e-3, weight_decay=0.01, state_bits=state_bits, seed=seed)
    gen = torch.Generator(device="cuda").manual_seed(seed)
    losses = []
    for step in range(steps):
        loss = loss_of(model, batch(gen, size, length, vocab))
        loss.backward()
        optimizer.step()
        optimizer.zero_grad(set_to_none=True)
        losses.append(loss.detach())
        if log and (step % 50 == 0 or step == steps - 1):
            log(f"step {step:4d}  loss {float(losses[-1]):.4f}")
    return [float(x) for x in losses]


if __name__ == "__main__":
    ap = argparse.ArgumentParser(description=__doc__, formatter_class=argparse.RawDescriptionHelpFormatter)
    for name, default in (("steps", 300), ("width", 256), ("layers", 2), ("length", 128), ("state-bits", 8)):
        ap.add_argument("--" + name, type=int, default=default)
    a = ap.parse_args()
    before = fb.fewbit_launch_count()
    train(a.steps, a.width, a.layers, a.length, state_bits=a.state_bits, log=print)
    print(f"{fb.fewbit_launch_count() - before} kernels of the library, {torch.cuda.max_memory_allocated() / 2 ** 20:.0f} MiB at most")
