"""A complete training step around the head, on synthetic data: token ids in, updated parameters out.

    python -m paper_2410_17765_b200.train_demo [--steps 60] [--bits 8]

The model is the smallest one that uses every operator as a trunk would: a tied embedding table, a norm, one gated block
(a matrix product, in place of attention or an MLP), its norms and residual addition, and the multi-token head.  The data
is a noisy walk over the vocabulary, so the loss has somewhere to go.  Everything but the block's three matrix products
runs in the library's kernels; nothing waits for the host within a step.
"""
from __future__ import annotations

import argparse
import math
from dataclasses import dataclass
from typing import Optional

import torch

from . import binding


@dataclass(frozen=True)
class Config:
    """Sequences per batch, tokens per sequence, width, vocabulary, predicted tokens, experts."""

    batch: int = 16
    length: int = 68
    d: int = 256
    V: int = 1024
    n: int = 3
    r: int = 4
    aux_coef: float = 0.01

    @property
    def positions(self) -> int:
        return self.batch * (self.length - self.n)


def walk(cfg: Config, generator: torch.Generator, follow: float = 0.9) -> torch.Tensor:
    """[batch, length] int32 tokens: the next one is 7 x + 3 (mod V) with probability `follow`, else any."""
    x = torch.randint(0, cfg.V, (cfg.batch, cfg.length), generator=generator, device="cuda")
    jump = torch.rand(cfg.batch, cfg.length, generator=generator, device="cuda") >= follow
    for t in range(1, cfg.length):
        x[:, t] = torch.where(jump[:, t], x[:, t], (7 * x[:, t - 1] + 3) % cfg.V)
    return x.to(torch.int32)


class Model:
    """Parameters, their gradients and the step.  Buffers that a step needs are made once, so that a step can be captured in a CUDA graph; one
    that is to be replayed as the next steps takes its number and rate from a binding.StepClock."""

    names = ("E", "w_in", "W_block", "w_post", "w_pre", "W_head", "W_g")

    def __init__(self, cfg: Config, seed: int = 0, *, bits: int = 8, master: bool = False):
        self.cfg = cfg
        gen = torch.Generator(device="cuda").manual_seed(seed)
        d, K = cfg.d, cfg.n * cfg.r

        def randn(*shape, std=0.02):
            return (torch.randn(*shape, generator=gen, device="cuda") * std).to(torch.bfloat16)

        self.E = randn(cfg.V, d)
        self.w_in, self.w_post, self.w_pre = (torch.ones(d, dtype=torch.bfloat16, device="cuda") for _ in range(3))
        self.W_block = randn(2 * d, d, std=1 / math.sqrt(d))                  # output and gate, one product
        self.W_head = randn(K, d, d, std=0.5 / math.sqrt(d))
        self.W_g = randn(cfg.r, d)
        self.grads = {k: torch.zeros_like(getattr(self, k)) for k in self.names}
        N = cfg.positions
        shape = binding.make_shape(N, d, cfg.V, cfg.n, cfg.r, cfg.aux_coef)
        self.saved = binding.Saved.alloc(shape)
        self.ws_head = binding.alloc_workspace(max(binding.workspace_bytes(shape, op) for op in (binding.OP_FORWARD, binding.OP_BACKWARD)))
        self.ws_embed = binding.alloc_workspace(binding.embed_workspace_bytes(N, cfg.V, d))
        self.ws_norm = binding.alloc_workspace(binding.norm_workspace_bytes(N, d))
        self.ws_clip = binding.alloc_workspace(binding.grad_norm_workspace_bytes([self.grads[k] for k in self.names]))
        self.status = torch.zeros(1, dtype=torch.int32, device="cuda")
        params = [getattr(self, k) for k in self.names]
        decay = [0.0 if p.dim() == 1 else 1.0 for p in params]                # norm weights are not decayed
        self.optimizer = binding.AdamW(params, bits=bits, master=master, decay_scale=decay)

    def forward(self, tokens: torch.Tensor) -> dict:
        """Loss and what the backward pass needs, for [positions] tokens and the [positions, n] that follow them."""
        c = self.cfg
        cur = tokens[:, :c.length - c.n].reshape(-1).contiguous()
        targets = torch.stack([tokens[:, s + 1:c.length - c.n + s + 1].reshape(-1) for s in range(c.n)], 1).contiguous()
        # fp32 residual stream
        x0 = binding.embed_forward(self.E, cur, scale=math.sqrt(c.d), out_dtype=torch.float32, dev_status=self.status)
        first = binding.norm_forward(x0, self.w_in)
        both = first["y"] @ self.W_block.t()
        block, gate = both[:, :c.d], both[:, c.d:]
        last = binding.norm_forward(x0, self.w_pre, block=block, gate=gate, w_post=self.w_post)
        head = binding.forward(last["y"], self.W_head, self.E, self.W_g, targets, aux_coef=c.aux_coef, saved=self.saved,
                               workspace=self.ws_head, dev_status=self.status)
        return dict(cur=cur, targets=targets, x0=x0, first=first, block=block, gate=gate, last=last, loss=head["loss"])

    def backward(self, f: dict) -> dict:
        """Gradients of the loss, into self.grads."""
        c, g = self.cfg, self.grads
        head = binding.backward(f["last"]["y"], self.W_head, self.E, self.W_g, f["targets"], self.saved, aux_coef=c.aux_coef,
                                workspace=self.ws_head, dev_status=self.status, out=dict(dW_head=g["W_head"], dE=g["E"], dW_g=g["W_g"]))
        both = torch.empty((c.positions, 2 * c.d), dtype=torch.bfloat16, device="cuda")
        last = binding.norm_backward(head["dh"], f["last"]["x_out"], self.w_pre, f["last"]["rstd_pre"], block=f["block"], gate=f["gate"],
                                     w_post=self.w_post, rstd_post=f["last"]["rstd_post"], workspace=self.ws_norm,
                                     out=dict(dblock=both[:, :c.d], dgate=both[:, c.d:], dw_post=g["w_post"], dw_pre=g["w_pre"]))
        torch.matmul(both.t(), f["first"]["y"], out=g["W_block"])
        first = binding.norm_backward(both @ self.W_block, f["x0"], self.w_in, f["first"]["rstd_pre"], dx_out=last["dx"],
                                      workspace=self.ws_norm, out=dict(dx=last["dx"], dw_pre=g["w_in"]))
        # the table is tied: its second gradient is added to the head's
        binding.embed_backward(first["dx"], f["cur"], c.V, scale=math.sqrt(c.d), out=g["E"], accumulate=True, workspace=self.ws_embed,
                               dev_status=self.status)
        return g

    def step(self, tokens: torch.Tensor, t, *, lr: Optional[float] = None, max_norm: float = 1.0) -> dict:
        """One optimiser step (the t-th, from 1, or a StepClock's next): {"loss", "norm"} on the device."""
        f = self.forward(tokens)
        g = self.backward(f)
        grads = [g[k] for k in self.names]
        clip = binding.grad_norm(grads, max_norm=max_norm, workspace=self.ws_clip)
        self.optimizer.step(grads, t, lr=lr, coef=clip["coef"], seed=0 if isinstance(t, binding.StepClock) else t)
        return dict(loss=f["loss"], norm=clip["norm"])


def train(steps: int = 60, *, cfg: Config = Config(), seed: int = 0, lr: float = 3e-3, bits: int = 8, master: bool = False) -> list:
    """Losses (nats per position, over n tokens) of `steps` steps."""
    model = Model(cfg, seed, bits=bits, master=master)
    gen = torch.Generator(device="cuda").manual_seed(seed + 1)
    losses = [model.step(walk(cfg, gen), t, lr=lr * min(1.0, t / 10))["loss"] for t in range(1, steps + 1)]
    if int(model.status.item()) != 0:
        raise binding.CpmtpError(f"cpmtp: device status {int(model.status.item())}")
    return [float(x) for x in losses]


def main() -> None:
    p = argparse.ArgumentParser(description=__doc__, formatter_class=argparse.RawDescriptionHelpFormatter)
    p.add_argument("--steps", type=int, default=60)
    p.add_argument("--bits", type=int, default=8, choices=(8, 32), help="optimiser states")
    p.add_argument("--master", action="store_true", help="keep fp32 copies of the parameters")
    p.add_argument("--lr", type=float, default=3e-3)
    a = p.parse_args()
    losses = train(a.steps, lr=a.lr, bits=a.bits, master=a.master)
    for t in sorted({0, *range(9, a.steps, 10), a.steps - 1}):
        print(f"step {t + 1:4d}  loss {losses[t]:.4f}")


if __name__ == "__main__":
    main()
