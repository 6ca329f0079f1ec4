"""Cases for the operators of the base model's pass over a draft: appending to a paged cache of keys and values, attention of a
few new tokens over it, eviction from it by accumulated attention weight, and sampling from logits.

`own` false: plain torch operations in 32 bits (sampling: in 64, where the border of a filter or of a drawn number matters).
`own` true: the library's entry points."""
import math
import random

import torch

own = False

BF16, F32 = "bf16", "f32"
DTYPE = {BF16: torch.bfloat16, F32: torch.float32}
INF = float("inf")


def listed():
    return [
        # a draft of four tokens and the one before it, eight positions, into pages of 64; keys and values are slices of one projection
        dict(name="append draft", op="append", B=8, Q=5, Hq=32, Hkv=8, D=128, page=64, most=4096, layout="NHD", acc=True, short=True),
        # four prompts of up to 2048 tokens
        dict(name="append prompt", op="append", B=4, Q=2048, Hq=32, Hkv=8, D=128, page=64, most=4096, layout="HND", acc=False, short=True),
        # one sequence, one new token, a short context: what a single user waits for
        dict(name="attend one", op="attend", B=1, Q=1, Hq=32, Hkv=8, D=128, page=64, most=1024, layout="NHD", acc=False, short=False, lse=True),
        # ordinary decoding: 64 sequences of ragged lengths, small pages
        dict(name="attend batch", op="attend", B=64, Q=1, Hq=32, Hkv=8, D=128, page=16, most=8192, layout="HND", acc=False, short=False, lse=False),
        # verification of drafts of up to four tokens, with the weights that eviction goes by
        dict(name="attend draft", op="attend", B=16, Q=5, Hq=32, Hkv=8, D=128, page=64, most=4096, layout="NHD", acc=True, short=True, lse=False),
        # two long contexts
        dict(name="attend long", op="attend", B=2, Q=1, Hq=64, Hkv=8, D=128, page=256, most=131072, layout="HND", acc=False, short=False, lse=True),
        # heads of their own, a width that no tile divides, pages that end inside a tile
        dict(name="attend odd", op="attend", B=7, Q=2, Hq=15, Hkv=5, D=80, page=24, most=5000, layout="NHD", acc=True, short=True, lse=True),
        # a batch that has outgrown its budget by four pages
        dict(name="evict batch", op="evict", B=16, Hkv=8, D=128, page=64, most=4352, budget=4096, recent=256, layout="NHD"),
        # two long prompts cut down
        dict(name="evict prompt", op="evict", B=2, Hkv=8, D=128, page=64, most=65536, budget=2048, recent=128, layout="HND"),
        # the base model's logits at eight positions, one setting for all of them
        dict(name="sample few", op="sample", N=8, V=128256, dtype=BF16, T=0.8, k=50, p=0.95, min_p=0.0, mixed=False, given=False),
        # a large batch of requests with settings of their own, greedy ones among them; log-probabilities of drafted tokens too
        dict(name="sample batch", op="sample", N=512, V=128256, dtype=F32, T=0.9, k=0, p=0.9, min_p=0.0, mixed=True, given=True),
        # an odd vocabulary, no filter but min-p
        dict(name="sample odd", op="sample", N=99, V=32003, dtype=BF16, T=1.3, k=0, p=1.0, min_p=0.02, mixed=False, given=True),
    ]


def _log(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    op = rng.choice(["append", "attend", "attend", "attend", "evict", "sample", "sample"])
    if op == "sample":
        N = _log(rng, 1, 512)
        V = _log(rng, 100, min(262144, 512 * 128256 // N))
        return dict(op=op, N=N, V=V, dtype=rng.choice([BF16, F32]), T=rng.choice([0.0, 0.3, 0.7, 1.0, 1.5]), k=rng.choice([0, 0, 1, 20, 64, 1000]),
                    p=rng.choice([1.0, 0.95, 0.8, 0.5]), min_p=rng.choice([0.0, 0.0, 0.01, 0.1]), mixed=rng.random() < 0.5, given=rng.random() < 0.5)
    Hkv, D, page, layout = rng.choice([1, 2, 4, 5, 8]), rng.choice([64, 80, 96, 128]), rng.choice([8, 16, 24, 64, 128, 256]), rng.choice(["NHD", "HND"])
    row = Hkv * D * 4
    if op == "append":
        B = _log(rng, 1, 64)
        Q = _log(rng, 1, min(4096, 8192 // B))
        return dict(op=op, B=B, Q=Q, Hq=Hkv * rng.choice([1, 4]), Hkv=Hkv, D=D, page=page, most=_log(rng, Q, 8192), layout=layout,
                    acc=rng.random() < 0.5, short=rng.random() < 0.5)
    if op == "evict":
        B = _log(rng, 1, 32)
        budget = _log(rng, 16, 4096)
        while B * budget * row > (1 << 28):
            B = B // 2
        most = _log(rng, budget // 2 + 1, min(65536, max(budget, (1 << 28) // (B * row))))
        return dict(op=op, B=B, Hkv=Hkv, D=D, page=page, most=most, budget=budget, recent=rng.randint(0, budget), layout=layout)
    B = _log(rng, 1, 64)
    most = _log(rng, 1, max(1, min(131072, (1 << 29) // (B * row))))
    Q = rng.choice([1, 1, 2, 5, 9])
    return dict(op=op, B=B, Q=Q, Hq=Hkv * rng.choice([1, 2, 4, 7, 8]), Hkv=Hkv, D=D, page=page, most=max(most, Q), layout=layout, acc=rng.random() < 0.4,
                short=rng.random() < 0.5, lse=rng.random() < 0.5)


def _lengths(case):
    """(slots, new tokens) of every sequence, the new ones included; the first sequence is the longest."""
    B, most, Q = case["B"], case["most"], case.get("Q", 0)
    r = random.Random(B * 1000003 + most * 31 + Q)
    news = [Q] + [r.randint(1, Q) if case.get("short") else Q for _ in range(B - 1)]
    lens = [most] + [max(n, int(most * r.uniform(0.3, 1.0))) for n in news[1:]]
    return lens, news


# ------------------------------------------------------------------------------------------------ inputs

def prepare(case, seed):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(int(seed) * 2654435761 % (1 << 62))
    s = dict(case=case)
    op = case["op"]

    def rand(*shape):
        return torch.rand(*shape, generator=gen, device="cuda")

    def randn(*shape, std=1.0):
        return torch.randn(*shape, generator=gen, device="cuda").mul_(std).to(torch.bfloat16)

    def ints(v):
        return torch.tensor(v, dtype=torch.int32, device="cuda")

    if op == "sample":
        N, V = case["N"], case["V"]
        s["logits"] = torch.randn(N, V, generator=gen, device="cuda").mul_(2.5).to(DTYPE[case["dtype"]])
        s["uniform"] = rand(N)
        for name, key, dtype in (("temperature", "T", torch.float32), ("top_k", "k", torch.int32), ("top_p", "p", torch.float32), ("min_p", "min_p", torch.float32)):
            s[name] = case[key]
            if case["mixed"]:      # every request its own; a few are greedy, a few have no filter at all
                kind = rand(N)
                one = torch.full((N,), case[key], dtype=torch.float32, device="cuda")
                other = {"T": rand(N) + 0.3, "k": (rand(N) * 100).floor() + 1, "p": rand(N) * 0.5 + 0.5, "min_p": rand(N) * 0.05}[key]
                off = {"T": 0.0, "k": 0.0, "p": 1.0, "min_p": 0.0}[key]
                s[name] = torch.where(kind < 0.5, one, torch.where(kind < 0.9, other, torch.full_like(one, off))).to(dtype)
        s["given"] = None
        if case["given"]:
            # drafted tokens: mostly likely ones
            likely = s["logits"].argmax(1)
            s["given"] = torch.where(rand(N) < 0.7, likely, (rand(N) * V).long().clamp_(max=V - 1)).to(torch.int32)
        return s
    B, Hkv, D, page = case["B"], case["Hkv"], case["D"], case["page"]
    lens, news = _lengths(case)
    pages = -(-max(lens) // page)
    more = -(-case["budget"] // page) if op == "evict" else 0
    P = B * (pages + more) + 3
    place = torch.randperm(P, generator=gen, device="cuda")[:B * (pages + more)].to(torch.int32).view(B, pages + more)
    s["table"] = place[:, :pages].contiguous()
    s["lens"] = ints(lens)
    for name in ("k_cache", "v_cache"):
        t = randn(P, page, Hkv, D) if case["layout"] == "NHD" else randn(P, Hkv, page, D).transpose(1, 2)
        s[name] = t
    s["acc"] = torch.randn(P, Hkv, page, generator=gen, device="cuda").mul_(2.0).exp_() if op == "evict" or case["acc"] else None
    if own:
        from paper_2410_17765_b200 import binding

        s["cache"] = binding.PagedCache(s["k_cache"], s["v_cache"], s["acc"])      # the handle that a server keeps
    if op == "evict":
        # some slots have not been looked at yet
        s["acc"].mul_(rand(P, Hkv, page) > 0.05)
        s["table_out"] = place[:, pages:].contiguous()
        return s
    Q, Hq = case["Q"], case["Hq"]
    s["q_lens"] = ints(news) if case["short"] else None
    both = randn(B, Q, (Hq + 2 * Hkv) * D)      # queries, keys and values of one projection
    if op == "append":
        s["k"] = both[:, :, Hq * D:(Hq + Hkv) * D].view(B, Q, Hkv, D)
        s["v"] = both[:, :, (Hq + Hkv) * D:].view(B, Q, Hkv, D)
        return s
    s["q"] = (both * 1.5)[:, :, :Hq * D].view(B, Q, Hq, D)
    s["out"] = torch.zeros(B, Q, Hq, D, dtype=torch.bfloat16, device="cuda")
    s["lse"] = torch.zeros(B, Q, Hq, device="cuda") if case["lse"] else None
    if own:
        s["workspace"] = binding.alloc_workspace(binding.cache_attend_workspace_bytes(s["cache"], B, pages, Q, Hq))
    return s


# ------------------------------------------------------------------------------------------------ plain forms

def _news(s):
    c = s["case"]
    return torch.full((c["B"],), c["Q"], device="cuda") if s["q_lens"] is None else s["q_lens"].long()


def _slots(t, slot):
    """Pages and places of slots [B, n] of the sequences of the table t."""
    page = slot // t[1]
    return t[0].long().gather(1, page.clamp(min=0, max=t[0].shape[1] - 1)), slot % t[1]


def _append(s):
    c = s["case"]
    news = _news(s).unsqueeze(1)
    j = torch.arange(c["Q"], device="cuda").unsqueeze(0)
    slot = s["lens"].long().unsqueeze(1) - news + j
    b, row = (j < news).nonzero(as_tuple=True)
    page, at = _slots((s["table"], c["page"]), slot)
    page, at = page[b, row], at[b, row]
    s["k_cache"][page, at] = s["k"][b, row]
    s["v_cache"][page, at] = s["v"][b, row]
    r = dict(k=s["k_cache"], v=s["v_cache"])
    if s["acc"] is not None:
        s["acc"][page, :, at] = 0.0
        r["acc"] = s["acc"]
    return r


def _whole(cache, table):
    """[B, slots, heads, D] of a cache in pages, in fp32."""
    B, n = table.shape
    return cache[table.long()].reshape(B, n * cache.shape[1], cache.shape[2], cache.shape[3]).float()


def _attend(s):
    c = s["case"]
    B, Q, Hkv, D = c["B"], c["Q"], c["Hkv"], c["D"]
    G = c["Hq"] // Hkv
    K, V = _whole(s["k_cache"], s["table"]), _whole(s["v_cache"], s["table"])
    S = K.shape[1]
    q = s["q"].float().view(B, Q, Hkv, G, D)
    score = torch.einsum("bqhgd,bshd->bhqgs", q, K) * (1.0 / math.sqrt(D))
    news, j = _news(s).unsqueeze(1), torch.arange(Q, device="cuda").unsqueeze(0)
    last = s["lens"].long().unsqueeze(1) - (news - 1 - j)                                     # [B, Q]: slots that a token sees
    row = j < news
    seen = (torch.arange(S, device="cuda") < last.unsqueeze(2)) & row.unsqueeze(2)             # [B, Q, S]
    score = score.masked_fill(~seen.view(B, 1, Q, 1, S), -INF)
    m = score.amax(4, keepdim=True).clamp(min=-3e38)
    e = torch.exp(score - m)
    total = e.sum(4, keepdim=True)
    p = e / total.clamp(min=1e-37)
    out = torch.einsum("bhqgs,bshd->bqhgd", p, V).reshape(B, Q, Hkv * G, D).to(torch.bfloat16)
    s["out"].copy_(torch.where(row.view(B, Q, 1, 1), out, s["out"]))
    r = dict(out=s["out"])
    if c["lse"]:
        lse = (m + torch.log(total)).view(B, Hkv, Q, G).transpose(1, 2).reshape(B, Q, Hkv * G)
        r["lse"] = s["lse"].copy_(torch.where(row.unsqueeze(2), lse, s["lse"]))
    if c["acc"]:
        w = p.sum((2, 3)).view(B, Hkv, -1, c["page"]).transpose(1, 2)                         # [B, pages, heads, page]
        s["acc"].index_add_(0, s["table"].long().view(-1), w.reshape(-1, Hkv, c["page"]))
        r["acc"] = s["acc"]
    return r


def _evict(s):
    c = s["case"]
    B, H, page, budget, recent = c["B"], c["Hkv"], c["page"], c["budget"], c["recent"]
    lens = s["lens"].long().view(B, 1, 1)
    key = s["acc"][s["table"].long()].transpose(1, 2).reshape(B, H, -1)
    slot = torch.arange(key.shape[2], device="cuda")
    key = torch.where(slot >= lens, -INF, torch.where(slot >= lens - recent, INF, key))
    order = key.sort(dim=2, descending=True, stable=True).indices
    if order.shape[2] < budget:
        order = torch.nn.functional.pad(order, (0, budget - order.shape[2]), value=1 << 30)
    at = torch.arange(budget, device="cuda")
    kept = torch.where((at < lens) & (order[:, :, :budget] < lens), order[:, :, :budget], 1 << 30).sort(2).values     # in order of the slots
    b, h, to = (at < lens).expand(B, H, budget).nonzero(as_tuple=True)
    frm = kept[b, h, to]
    src = s["table"].long()[b, frm // page]
    dst = s["table_out"].long()[b, to // page]
    for cache in (s["k_cache"], s["v_cache"]):
        cache[dst, to % page, h] = cache[src, frm % page, h]
    s["acc"][dst, h, to % page] = s["acc"][src, h, frm % page]
    kept = torch.where(kept == 1 << 30, -1, kept).to(torch.int32)
    return dict(k=s["k_cache"], v=s["v_cache"], acc=s["acc"], lens=s["lens"].clamp(max=budget), kept=kept)


def _column(v, N, dtype):
    return v.to(dtype).view(N, 1) if torch.is_tensor(v) else torch.full((N, 1), v, dtype=torch.float32, device="cuda").to(dtype)


def _sample(s):
    N, V = s["logits"].shape
    T, k = _column(s["temperature"], N, torch.float64), _column(s["top_k"], N, torch.int64)
    p, min_p = _column(s["top_p"], N, torch.float64), _column(s["min_p"], N, torch.float64)
    x = s["logits"].float()
    order = x.sort(dim=1, descending=True, stable=True).indices
    k = torch.where(k > 0, k, V)
    k = torch.where(T > 0, k, 1)
    x = x.double()
    z = (x - x.amax(1, keepdim=True)) / torch.where(T > 0, T, 1.0)
    w = torch.exp(z)
    rank = torch.arange(V, device="cuda")
    ranked = w.gather(1, order) * (rank < k)
    before = ranked.cumsum(1) - ranked
    keep = (rank < k) & ((before < p * ranked.sum(1, keepdim=True)) | (rank == 0) | (p >= 1)) & ((ranked >= min_p) | (rank == 0))
    kept = torch.zeros_like(keep).scatter_(1, order, keep)
    w = w * kept
    run_sum = w.cumsum(1)
    total = run_sum[:, -1:]
    over = (run_sum > s["uniform"].double().view(N, 1) * total) & kept
    token = over.to(torch.int8).argmax(1, keepdim=True)
    logp = (z.gather(1, token) - torch.log(total)).view(N).float()
    r = dict(tokens=token.view(N).to(torch.int32), logp=logp, kept=kept.sum(1).to(torch.int32))
    if s["given"] is not None:
        g = s["given"].long().view(N, 1)
        r["logp_given"] = torch.where(kept.gather(1, g), z.gather(1, g) - torch.log(total), -INF).view(N).float()
    return r


# ------------------------------------------------------------------------------------------------ one pass

def run(s):
    c = s["case"]
    op = c["op"]
    if not own:
        return {"append": _append, "attend": _attend, "evict": _evict, "sample": _sample}[op](s)
    from paper_2410_17765_b200 import binding

    if op == "append":
        binding.cache_append(s["cache"], s["k"], s["v"], s["table"], s["lens"], q_lens=s["q_lens"])
        r = dict(k=s["k_cache"], v=s["v_cache"])
        if s["acc"] is not None:
            r["acc"] = s["acc"]
        return r
    if op == "attend":
        r = dict(out=s["out"])
        if c["lse"]:
            r["lse"] = s["lse"]
        binding.cache_attend(s["cache"], s["q"], s["table"], s["lens"], q_lens=s["q_lens"], out=r, workspace=s["workspace"])
        if c["acc"]:
            r["acc"] = s["acc"]
        return r
    if op == "evict":
        r = binding.cache_evict(s["cache"], s["table"], s["lens"], s["table_out"], c["budget"], recent=c["recent"])
        return dict(k=s["k_cache"], v=s["v_cache"], acc=s["acc"], lens=r["lens"], kept=r["kept"])
    return binding.sample_logits(s["logits"], s["uniform"], temperature=s["temperature"], top_k=s["top_k"], top_p=s["top_p"], min_p=s["min_p"],
                                 given=s["given"], want_kept=True)


def work(case):
    op = case["op"]
    if op == "sample":
        n = case["N"] * case["V"]
        return dict(bytes=n * (2 if case["dtype"] == BF16 else 4) + case["N"] * 32, flops=4 * n)
    lens, news = _lengths(case)
    H, D = case["Hkv"], case["D"]
    if op == "append":
        return dict(bytes=sum(news) * H * (8 * D + (4 if case["acc"] else 0)), flops=0)
    if op == "evict":
        kept = sum(min(n, case["budget"]) for n in lens)
        return dict(bytes=H * (4 * sum(lens) + kept * (8 * D + 8)), flops=H * sum(lens))
    rows = case["Hq"] * D * 4 * sum(news)
    return dict(bytes=sum(lens) * H * (4 * D + (8 if case["acc"] else 0)) + rows,
                flops=4 * D * case["Hq"] * sum(n * q for n, q in zip(lens, news)))


# ------------------------------------------------------------------------------------------------ in 64 bits

def exact(case, seed):
    """What run() returns, from the definitions, one sequence or row at a time."""
    s = prepare(case, seed)
    op = case["op"]
    if op == "append" or op == "evict":
        return None      # nothing is computed: values are moved
    if op == "sample":
        logits, N = s["logits"].double(), case["N"]
        setting = {k: s[k].tolist() if torch.is_tensor(s[k]) else [s[k]] * N for k in ("temperature", "top_k")}
        frac = {k: (s[k] if torch.is_tensor(s[k]) else torch.full((N,), s[k], device="cuda")).double().tolist() for k in ("top_p", "min_p")}
        logp, given = [], []
        for i in range(N):
            x, T = logits[i], setting["temperature"][i]
            top = torch.arange(case["V"], device="cuda")[x == x.max()][:1]
            if T == 0:
                mask = torch.zeros(case["V"], dtype=torch.bool, device="cuda")
                mask[top] = True
                T = 1.0
            else:
                T = float(torch.tensor(T, dtype=torch.float32).double())
                values, ids = torch.sort(x, descending=True, stable=True)
                n = setting["top_k"][i] or case["V"]
                values, ids = values[:n], ids[:n]
                mass = torch.exp((values - values[0]) / T)
                if frac["top_p"][i] < 1:
                    share = torch.cumsum(mass, 0) / mass.sum()
                    n = int((share < frac["top_p"][i]).sum()) + 1
                    mass, ids = mass[:n], ids[:n]
                ids = ids[mass >= frac["min_p"][i]] if frac["min_p"][i] <= 1 else ids[:1]
                mask = torch.zeros(case["V"], dtype=torch.bool, device="cuda")
                mask[ids] = True
            scaled = x / T
            norm = torch.logsumexp(scaled[mask], 0)
            e = torch.where(mask, torch.exp(scaled - norm), 0.0)
            cdf = torch.cumsum(e, 0)
            token = torch.nonzero((cdf > float(s["uniform"][i]) * cdf[-1]) & mask)[0, 0]
            logp.append(scaled[token] - norm)
            if s["given"] is not None:
                g = s["given"][i].long()
                given.append(torch.where(mask[g], scaled[g] - norm, -INF))
        r = dict(tokens=None, logp=torch.stack(logp), kept=None)
        if s["given"] is not None:
            r["logp_given"] = torch.stack(given)
        return r
    lens, news = _lengths(case)
    news = news if case["short"] else [case["Q"]] * case["B"]
    G, page = case["Hq"] // case["Hkv"], case["page"]
    out = s["out"].double()
    lse = torch.zeros(case["B"], case["Q"], case["Hq"], dtype=torch.float64, device="cuda")
    acc = s["acc"].double() if case["acc"] else None
    for b, (n, new) in enumerate(zip(lens, news)):
        place = s["table"][b].long().repeat_interleave(page)[:n]
        offset = torch.arange(n, device="cuda") % page
        K, V = s["k_cache"][place, offset].double(), s["v_cache"][place, offset].double()
        for j in range(new):
            seen = n - (new - 1 - j)
            dot = torch.matmul(s["q"][b, j].double().view(case["Hkv"], G, -1), K[:seen].permute(1, 2, 0)) / math.sqrt(case["D"])
            norm = torch.logsumexp(dot, 2)
            weight = torch.exp(dot - norm.unsqueeze(2))
            out[b, j] = torch.matmul(weight, V[:seen].transpose(0, 1)).reshape(case["Hq"], -1)
            lse[b, j] = norm.reshape(-1)
            if acc is not None:
                acc[place[:seen], :, offset[:seen]] += weight.sum(1).t()
    r = dict(out=out)
    if case["lse"]:
        r["lse"] = lse
    if case["acc"]:
        r["acc"] = acc
    return r
