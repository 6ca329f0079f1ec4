"""Drafting and verifying on synthetic weights: prompts in, tokens out.

    python -m paper_2410_17765_b200.serve_demo [--steps 40] [--temperature 0.8] [--top-p 0.95] [--budget 96]

The base model is a small pre-norm trunk with grouped-query attention and no position encoding; the multi-token head drafts from its hidden
states.  A round runs the base model once over the last token and the draft behind it: lookup, norms, attention over the paged cache that
the tokens have been appended to, logits, a token from each row.  The draft is kept as far as the base model agrees with it, the rejected
tokens' slots are given up by their length alone, and the base model's own token follows.  Every so often the cache is cut down to a
budget by the attention weight that its slots have received (from drafted tokens too that were not kept).  The matrix products between the library's kernels are torch's; nothing
waits for the host within a round.
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
    """Layers, width, query heads, cache heads, vocabulary, drafted tokens (the last known one included), experts, slots to a page."""

    layers: int = 2
    d: int = 256
    Hq: int = 4
    H: int = 2
    V: int = 1024
    n: int = 4
    r: int = 4
    page_slots: int = 16

    @property
    def D(self) -> int:
        return self.d // self.Hq


class Base:
    """Random weights of a trunk and of the head that drafts from it."""

    def __init__(self, cfg: Config, seed: int = 0):
        self.cfg = cfg
        gen = torch.Generator(device="cuda").manual_seed(seed)
        d = cfg.d

        def randn(*shape, std):
            return (torch.randn(*shape, generator=gen, device="cuda") * std).to(torch.bfloat16)

        self.E = randn(cfg.V, d, std=1.0 / math.sqrt(d))
        self.w_norm = [torch.ones(d, dtype=torch.bfloat16, device="cuda") for _ in range(cfg.layers + 1)]
        self.W_qkv = [randn((cfg.Hq + 2 * cfg.H) * cfg.D, d, std=1.5 / math.sqrt(d)) for _ in range(cfg.layers)]
        self.W_out = [randn(d, cfg.Hq * cfg.D, std=1.0 / math.sqrt(d)) for _ in range(cfg.layers)]
        self.W_head = randn(cfg.n * cfg.r, d, d, std=1.0 / math.sqrt(d))
        self.W_g = randn(cfg.r, d, std=0.02)


class Server:
    """Sequences under way: their pages, lengths and last tokens, all on the device."""

    def __init__(self, base: Base, batch: int, slots: int, *, budget: int = 0, recent: int = 0):
        c = base.cfg
        self.base, self.batch, self.budget, self.recent = base, batch, budget, recent
        self.width = -(-slots // c.page_slots)
        # two sets of pages to a sequence: eviction moves it from one to the other
        sets = 2 if budget else 1
        pages = batch * self.width * sets
        order = torch.randperm(pages, device="cuda").to(torch.int32).view(sets, batch, self.width)
        self.tables = [order[i].contiguous() for i in range(sets)]

        def cache():
            k, v = (torch.zeros(pages, c.page_slots, c.H, c.D, dtype=torch.bfloat16, device="cuda") for _ in range(2))
            return binding.PagedCache(k, v, torch.zeros(pages, c.H, c.page_slots, device="cuda") if budget else None)

        self.caches = [cache() for _ in range(c.layers)]
        self.lens = torch.zeros(batch, dtype=torch.int32, device="cuda")         # slots whose tokens are settled
        self.h = self.last = None                                                # hidden state that drafts; the token behind it
        self.status = torch.zeros(1, dtype=torch.int32, device="cuda")

    def forward(self, tokens: torch.Tensor, q_lens: Optional[torch.Tensor] = None) -> torch.Tensor:
        """Hidden states [batch, Q, d] of new tokens [batch, Q], whose keys and values join the cache behind lens."""
        c, b, st = self.base.cfg, self.base, dict(dev_status=self.status)
        B, Q = tokens.shape
        lens = self.lens + (Q if q_lens is None else q_lens)
        x = binding.embed_forward(b.E, tokens.contiguous(), scale=math.sqrt(c.d), out_dtype=torch.float32, **st).view(B * Q, c.d)
        y = binding.norm_forward(x, b.w_norm[0])["y"]
        for layer, cache in enumerate(self.caches):
            qkv = (y @ b.W_qkv[layer].t()).view(B, Q, c.Hq + 2 * c.H, c.D)
            q, k, v = qkv[:, :, :c.Hq], qkv[:, :, c.Hq:c.Hq + c.H], qkv[:, :, c.Hq + c.H:]
            binding.cache_append(cache, k, v, self.tables[0], lens, q_lens=q_lens, **st)
            out = binding.cache_attend(cache, q, self.tables[0], lens, q_lens=q_lens, **st)["out"]
            both = binding.norm_forward(x, b.w_norm[layer + 1], block=out.view(B * Q, c.Hq * c.D) @ b.W_out[layer].t())
            x, y = both["x_out"], both["y"]
        return y.view(B, Q, c.d)

    def sample(self, h: torch.Tensor, uniform: torch.Tensor, **how) -> dict:
        """Tokens from the base model's logits at hidden states [N, d]."""
        return binding.sample_logits(h @ self.base.E.t(), uniform, dev_status=self.status, **how)

    def start(self, prompts: torch.Tensor, lengths: torch.Tensor, uniform: torch.Tensor, **how) -> torch.Tensor:
        """Reads prompts [batch, T] of `lengths` tokens (int32); returns the first token behind each."""
        h = self.forward(prompts, lengths)
        self.lens = self.lens + lengths
        self.h = h[torch.arange(self.batch, device="cuda"), lengths.long() - 1].contiguous()
        self.last = self.sample(self.h, uniform, **how)["tokens"]
        return self.last

    def round(self, uniform: torch.Tensor, **how) -> tuple:
        """Drafts, verifies, and moves on: (tokens [batch, n] int32, how many of them each sequence has gained [batch] int32)."""
        c, b, B = self.base.cfg, self.base, self.batch
        forced = torch.full((B, c.n), -1, dtype=torch.int32, device="cuda")
        forced[:, 0] = self.last
        draft = binding.sample_draft(self.h, b.W_head, b.E, b.W_g, c.n, forced=forced, dev_status=self.status)["draft"]
        h = self.forward(draft)
        # the base model's token behind every token of the draft
        own = self.sample(h.view(B * c.n, c.d), uniform.view(-1), **how)["tokens"].view(B, c.n)
        kept = binding.verify_draft(draft[:, 1:].contiguous(), own[:, :c.n - 1].contiguous())
        rows = torch.arange(B, device="cuda")
        self.lens = self.lens + kept + 1
        self.h = h[rows, kept.long()].contiguous()
        self.last = own[rows, kept.long()].contiguous()
        return own, kept + 1

    def evict(self) -> None:
        """Cuts every sequence down to the budget."""
        for cache in self.caches:
            lens = binding.cache_evict(cache, self.tables[0], self.lens, self.tables[1], self.budget, recent=self.recent, dev_status=self.status)["lens"]
        self.tables.reverse()
        self.lens = lens


def generate(cfg: Config = Config(), *, batch: int = 8, prompt: int = 24, steps: int = 40, seed: int = 0, budget: int = 0, recent: int = 16,
             every: int = 8, **how) -> tuple:
    """(tokens of each sequence as lists, tokens gained per round) of `steps` rounds on random prompts of ragged lengths.
    Of a budget, the last `recent` slots stay whatever their weight; all of it where it is smaller."""
    gen = torch.Generator(device="cuda").manual_seed(seed + 1)
    slots = (budget + every * cfg.n if budget else prompt + steps * cfg.n) + cfg.n + prompt
    server = Server(Base(cfg, seed), batch, slots, budget=budget, recent=min(recent, budget))
    prompts = torch.randint(0, cfg.V, (batch, prompt), generator=gen, device="cuda").to(torch.int32)
    lengths = torch.randint(1, prompt + 1, (batch,), generator=gen, device="cuda").to(torch.int32)
    first = server.start(prompts, lengths, torch.rand(batch, generator=gen, device="cuda"), **how)
    rounds = []
    for i in range(steps):
        if budget and i % every == every - 1:
            server.evict()
        rounds.append(server.round(torch.rand(batch, cfg.n, generator=gen, device="cuda"), **how))
    if int(server.status.item()) != 0:
        raise binding.CpmtpError(f"cpmtp: device status {int(server.status.item())}")
    out = [[t] for t in first.tolist()]
    gained = 0
    for tokens, count in rounds:
        for b, (row, k) in enumerate(zip(tokens.tolist(), count.tolist())):
            out[b] += row[:k]
            gained += k
    return out, gained / (steps * batch)


def main() -> None:
    p = argparse.ArgumentParser(description=__doc__, formatter_class=argparse.RawDescriptionHelpFormatter)
    p.add_argument("--steps", type=int, default=40)
    p.add_argument("--batch", type=int, default=8)
    p.add_argument("--temperature", type=float, default=0.0)
    p.add_argument("--top-k", type=int, default=0)
    p.add_argument("--top-p", type=float, default=1.0)
    p.add_argument("--min-p", type=float, default=0.0)
    p.add_argument("--budget", type=int, default=0, help="slots that eviction leaves to a sequence (0: none is done)")
    a = p.parse_args()
    tokens, gained = generate(batch=a.batch, steps=a.steps, budget=a.budget, temperature=a.temperature, top_k=a.top_k, top_p=a.top_p, min_p=a.min_p)
    print(f"{sum(map(len, tokens))} tokens in {a.steps} rounds of {a.batch} sequences, {gained:.2f} a round and sequence (random weights)")


if __name__ == "__main__":
    main()
