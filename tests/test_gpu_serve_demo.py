"""The operators of the base model's pass over a draft together, as a server uses them."""
import math

import pytest
import torch

pytestmark = pytest.mark.gpu


def plain_hidden(base, tokens):
    """Hidden states [T, d] of one sequence in fp64, without a cache."""
    c = base.cfg

    def norm(x, w):
        return x * torch.rsqrt(x.square().mean(-1, keepdim=True) + 1e-6) * w.double()

    x = base.E.double()[tokens] * math.sqrt(c.d)
    T = len(tokens)
    seen = torch.ones(T, T, dtype=torch.bool, device="cuda").tril()
    y = norm(x, base.w_norm[0])
    for layer in range(c.layers):
        qkv = (y @ base.W_qkv[layer].double().t()).view(T, c.Hq + 2 * c.H, c.D)
        q, k, v = qkv[:, :c.Hq], qkv[:, c.Hq:c.Hq + c.H], qkv[:, c.Hq + c.H:]
        k, v = (t.repeat_interleave(c.Hq // c.H, 1) for t in (k, v))
        s = torch.einsum("qhd,khd->hqk", q, k) / math.sqrt(c.D)
        p = torch.softmax(s.masked_fill(~seen, -float("inf")), 2)
        x = x + torch.einsum("hqk,khd->qhd", p, v).reshape(T, c.Hq * c.D) @ base.W_out[layer].double().t()
        y = norm(x, base.w_norm[layer + 1])
    return y


@pytest.mark.parametrize("V", [1024, 4])
def test_rounds_follow_the_base_model(V):
    """Greedy: every token that a sequence gains is the one that the base model, computed without a cache and in fp64, ranks first after the tokens
    before it, or is ranked within the rounding of the bf16 intermediate results of it.  Those are: y, qkv, out and the block's output
    of each layer, and the logits, 2^-8 of their values each, nine in a row: 9 x 2^-8 of a hidden state's norm in the worst case, and so
    of a logit's spread, |h| |E_v| (sqrt(d) x 1, as rows of E have norm 1).  The hidden states that the last round left are compared by that norm
    too."""
    from paper_2410_17765_b200 import serve_demo as S

    cfg = S.Config(V=V)
    tol = 9 * 2.0 ** -8 * math.sqrt(cfg.d)
    base = S.Base(cfg, 3)
    gen = torch.Generator(device="cuda").manual_seed(4)
    B, T = 4, 20
    server = S.Server(base, B, 80)
    prompts = torch.randint(0, cfg.V, (B, T), generator=gen, device="cuda").to(torch.int32)
    lengths = torch.tensor([20, 1, 7, 16], dtype=torch.int32, device="cuda")
    u = torch.zeros(B, cfg.n, device="cuda")
    seqs = [prompts[b, :n].tolist() for b, n in enumerate(lengths.tolist())]
    first = server.start(prompts, lengths, u[:, 0].contiguous(), temperature=0.0)
    starts = [len(s) for s in seqs]
    for b, t in enumerate(first.tolist()):
        seqs[b].append(t)
    for _ in range(6):
        tokens, gained = server.round(u, temperature=0.0)
        for b, (row, k) in enumerate(zip(tokens.tolist(), gained.tolist())):
            assert 1 <= k <= cfg.n
            seqs[b] += row[:k]
    assert int(server.status.item()) == 0
    assert server.lens.tolist() == [len(s) - 1 for s in seqs]
    for s, start in zip(seqs, starts):
        logits = plain_hidden(base, torch.tensor(s[:-1], device="cuda")) @ base.E.double().t()
        hidden = plain_hidden(base, torch.tensor(s[:-1], device="cuda"))[-1]
        got = server.h[seqs.index(s)].double()
        assert float((got - hidden).norm()) <= 9 * 2.0 ** -8 * float(hidden.norm())
        for i in range(start, len(s)):
            row = logits[i - 1]
            assert float(row.max() - row[s[i]]) <= 2 * tol, (i, float(row.max() - row[s[i]]))


def test_drafts_that_are_right_are_kept(monkeypatch):
    """Drafts that foretell what the base model says, and then go wrong: their tokens are kept up to there, and the sequence goes on."""
    from paper_2410_17765_b200 import binding, serve_demo as S

    cfg = S.Config()
    base = S.Base(cfg, 7)
    prompts = torch.arange(60, dtype=torch.int32, device="cuda").view(3, 20)
    lengths, u = torch.full((3,), 20, dtype=torch.int32, device="cuda"), torch.zeros(3, cfg.n, device="cuda")

    def run(rounds):
        server = S.Server(base, 3, 120)
        out = [[t] for t in server.start(prompts, lengths, u[:, 0].contiguous(), temperature=0.0).tolist()]
        counts = []
        for _ in range(rounds):
            tokens, gained = server.round(u, temperature=0.0)
            counts.append(gained.tolist())
            for s, row, k in zip(out, tokens.tolist(), gained.tolist()):
                s += row[:k]
        assert int(server.status.item()) == 0 and server.lens.tolist() == [19 + len(s) for s in out]
        return out, counts

    plain, _ = run(24)
    at = [0, 0, 0]                                            # the last known token of each sequence
    right = [cfg.n - 1, 1, 0]                                 # drafted tokens that are right

    def foretold(h, *args, forced, **kw):
        rows = [plain[b][i:i + 1 + right[b]] + [(plain[b][i + 1 + right[b]] + 1) % cfg.V] * (cfg.n - 1 - right[b]) for b, i in enumerate(at)]
        draft = torch.tensor(rows, dtype=torch.int32, device="cuda")
        assert torch.equal(draft[:, 0], forced[:, 0])
        for b in range(3):
            at[b] += 1 + right[b]
        return dict(draft=draft)

    monkeypatch.setattr(binding, "sample_draft", foretold)
    rounds = 4
    got, counts = run(rounds)
    assert all(c == [1 + k for k in right] for c in counts)
    assert all(g == p[:len(g)] for g, p in zip(got, plain))


@pytest.mark.parametrize("how", [dict(temperature=0.0), dict(temperature=0.9, top_p=0.9), dict(temperature=0.7, top_k=20, min_p=0.02)])
@pytest.mark.parametrize("budget", [0, 40])
def test_generation_repeats(how, budget):
    from paper_2410_17765_b200 import serve_demo as S

    a, gained = S.generate(steps=20, budget=budget, **how)
    b, _ = S.generate(steps=20, budget=budget, **how)
    assert a == b and 1.0 <= gained <= S.Config().n
    assert all(0 <= t < S.Config().V for s in a for t in s)
    if budget == 0:
        assert all(len(s) >= 21 for s in a)


def test_eviction_within_the_budget_changes_nothing():
    """A budget that no sequence reaches moves the cache to other pages and leaves every token as it was."""
    from paper_2410_17765_b200 import serve_demo as S

    plain, _ = S.generate(steps=16, temperature=0.0)
    moved, _ = S.generate(steps=16, temperature=0.0, budget=512, every=5)
    assert plain == moved
