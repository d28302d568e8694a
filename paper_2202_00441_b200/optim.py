"""AdamW with moments of 8 (or 32) bits as a PyTorch optimizer over ``fewbit_adamw_step``."""
from __future__ import annotations

import torch

from .operators import ADAMW_BLOCK, fewbit_adamw_create, fewbit_adamw_step


def _mix(x: int) -> int:
    """The 64-bit finaliser of SplitMix64 (Steele, Lea and Flood, Fast splittable pseudorandom number generators, 2014)."""
    x = (x + 0x9E3779B97F4A7C15) & 0xFFFFFFFFFFFFFFFF
    x = ((x ^ (x >> 30)) * 0xBF58476D1CE4E5B9) & 0xFFFFFFFFFFFFFFFF
    x = ((x ^ (x >> 27)) * 0x94D049BB133111EB) & 0xFFFFFFFFFFFFFFFF
    return x ^ (x >> 31)


def _noise_seed(*parts: int) -> int:
    """32 bits for one call's stochastic rounding.  The library's noise for a place is a hash of place * odd constant + seed: all
    seeds' noise is one sequence of 2^32 values that starts at different places.  A seed that grew by a fixed amount each step
    would start next to the last one's; mixed ones start anywhere."""
    x = 0
    for part in parts:
        x = _mix(x ^ (part & 0xFFFFFFFFFFFFFFFF))
    return x >> 32


class FewBitAdamW(torch.optim.Optimizer):
    """Drop-in for ``torch.optim.AdamW`` on CUDA parameters of float32, bfloat16 or float16.

    state_bits: 8 keeps each moment as one float8 code an element and one float32 scale for each 256 elements (rounded
    stochastically, from ``seed``), 32 keeps float32 moments.  master: 16-bit parameters get a float32 copy that the step
    updates; the parameter is its rounding.  All parameters of one type and device are updated in one launch (up to 400
    tensors).  ``step(grad_scale=t)`` multiplies every gradient by the one float32 value ``t`` on the device."""

    def __init__(self, params, lr: float = 1e-3, betas=(0.9, 0.999), eps: float = 1e-8, weight_decay: float = 1e-2,
                 state_bits: int = 8, master: bool = True, seed: int = 0):
        if state_bits not in (8, 32):
            raise ValueError("state_bits must be 8 or 32")
        self._handles, self.seed = {}, int(seed)
        super().__init__(params, dict(lr=lr, betas=betas, eps=eps, weight_decay=weight_decay, state_bits=state_bits, master=master))

    def add_param_group(self, group):
        super().add_param_group(group)
        for p in self.param_groups[-1]["params"]:
            if not p.is_cuda or not p.is_contiguous() or p.dtype not in (torch.float32, torch.bfloat16, torch.float16):
                del self.param_groups[-1]
                raise ValueError("parameters must be contiguous CUDA tensors of float32, bfloat16 or float16")

    def __getstate__(self):
        return {**super().__getstate__(), "seed": self.seed}

    def __setstate__(self, state):
        super().__setstate__(state)
        self._handles = {}

    def load_state_dict(self, state_dict):
        super().load_state_dict(state_dict)
        # the base class converts floating state to the parameter's type; codes, scales and masters keep theirs
        for saved, group in zip(state_dict["param_groups"], self.param_groups):
            for key, p in zip(saved["params"], group["params"]):
                if key in state_dict["state"]:
                    self.state[p] = {k: v.to(p.device, copy=True) if torch.is_tensor(v) else v for k, v in state_dict["state"][key].items()}
        self._handles = {}

    def _init_state(self, p, group):
        state = self.state[p]
        state["step"] = 0
        if group["state_bits"] == 8:
            blocks = -(-p.numel() // ADAMW_BLOCK)
            for name in ("exp_avg", "exp_avg_sq"):
                state[name] = torch.zeros(p.shape, dtype=torch.uint8, device=p.device).view(torch.float8_e4m3fn)
                state[name + "_scale"] = torch.zeros(blocks, dtype=torch.float32, device=p.device)
        else:
            for name in ("exp_avg", "exp_avg_sq"):
                state[name] = torch.zeros(p.shape, dtype=torch.float32, device=p.device)
        if group["master"] and p.dtype != torch.float32:
            state["master"] = p.detach().float()

    @torch.no_grad()
    def step(self, closure=None, grad_scale: torch.Tensor | None = None):
        loss = None
        if closure is not None:
            with torch.enable_grad():
                loss = closure()
        for number, group in enumerate(self.param_groups):
            buckets = {}
            for index, p in enumerate(group["params"]):
                if p.grad is None:
                    continue
                if p.grad.is_sparse:
                    raise RuntimeError("FewBitAdamW takes dense gradients")
                if not self.state[p]:
                    self._init_state(p, group)
                buckets.setdefault((p.device, p.dtype, self.state[p]["step"]), []).append((index, p))
            for place, ((device, dtype, step), members) in enumerate(buckets.items()):
                params = [p for _, p in members]
                names = ["exp_avg", "exp_avg_sq"]
                if group["state_bits"] == 8:
                    names += ["exp_avg_scale", "exp_avg_sq_scale"]
                lists = [[self.state[p][n] for p in params] for n in names] + [None] * (4 - len(names))
                masters = [self.state[p]["master"] for p in params] if "master" in self.state[params[0]] else None
                # a handle for each set of parameters that step together; made anew when one of them or of their state is another tensor
                key = (number, tuple(i for i, _ in members))
                tensors = [t for x in [params, *lists, masters] if x is not None for t in x]
                held = self._handles.pop(key, None)
                if held is None or len(held[0]) != len(tensors) or any(a is not b for a, b in zip(held[0], tensors)):
                    held = (tensors, fewbit_adamw_create(params, *lists, masters))
                self._handles[key] = held
                if len(self._handles) > 64:                      # the one that has not been used for longest
                    del self._handles[next(iter(self._handles))]
                grads = [p.grad.to(dtype).contiguous() for p in params]
                fewbit_adamw_step(held[1], grads, step=step + 1, lr=float(group["lr"]), betas=group["betas"], eps=group["eps"],
                                  weight_decay=group["weight_decay"], seed=_noise_seed(self.seed, step + 1, number, place),
                                  grad_scale=grad_scale)
                for p in params:
                    self.state[p]["step"] = step + 1
        return loss
