"""Cases for the operators around the multi-token head in a training step: embedding lookup and its gradient, the
norms and gated residual addition around a block, and the AdamW step with gradient clipping.

`own` false: plain torch operations in 32 bits.  `own` true: the library's entry points."""
import math
import random

import torch

own = False

BF16, F32 = "bf16", "f32"
BLOCK = 256          # elements of an 8-bit state that share an exponent
DTYPE = {BF16: torch.bfloat16, F32: torch.float32}


def listed():
    return [
        # lookup of the tokens of a draft being verified: 8 positions x 4 tokens
        dict(name="embed fwd draft", op="embed_fwd", T=32, d=4096, V=128256, scale=1.0, out=BF16, pad=0.0),
        # a training batch of 8 sequences of 1024 tokens into an fp32 residual stream, scaled by sqrt(d)
        dict(name="embed fwd train", op="embed_fwd", T=8192, d=2048, V=32000, scale=math.sqrt(2048.0), out=F32, pad=0.02),
        # tied table: added to the dE that the head's backward pass wrote
        dict(name="embed bwd tied", op="embed_bwd", T=8192, d=4096, V=32000, scale=1.0, dy=BF16, accumulate=True, pad=0.0),
        # untied table of a large vocabulary: the whole dE is written, most of its rows are zero
        dict(name="embed bwd bigvocab", op="embed_bwd", T=16384, d=4096, V=128256, scale=1.0, dy=BF16, accumulate=False, pad=0.05),
        # one decode step of 8 positions through a block's norms; block output and gate are halves of one projection
        dict(name="norm fwd decode", op="norm_fwd", N=8, d=4096, stream=BF16, gate="channel", post=True, fused=True, res_scale=1.0),
        # the training step's positions at the width of the largest named workload
        dict(name="norm fwd train", op="norm_fwd", N=8192, d=4096, stream=BF16, gate="channel", post=True, fused=True, res_scale=1.0),
        dict(name="norm bwd train", op="norm_bwd", N=8192, d=4096, stream=BF16, gate="channel", post=True, fused=True, res_scale=1.0),
        # fp32 residual stream, one gate per position, a width and a row count that no vector or tile divides
        dict(name="norm bwd odd", op="norm_bwd", N=4099, d=1023, stream=F32, gate="row", post=True, fused=False, res_scale=0.70710678),
        # optimiser step of a small head (d = 256, V = 1024, n = 3, r = 4): three tensors, clipped, fp32 master copy
        dict(name="adamw tiny", op="adamw", sizes="head", n=3, r=4, d=256, V=1024, param=BF16, master=True, bits=32, clip=1.0),
        # sixty tensors of ragged sizes, fp32 parameters
        dict(name="adamw ragged", op="adamw", sizes="ragged", count=60, largest=400000, param=F32, master=False, bits=32, clip=1.0),
        # W_head, E and W_g at d = 2048, V = 32000, n = 2, r = 8, fp32 master copy, clipped
        dict(name="adamw train", op="adamw", sizes="head", n=2, r=8, d=2048, V=32000, param=BF16, master=True, bits=32, clip=1.0),
        # the same tensors at d = 4096, n = 4: states in 8 bits, bf16 parameters without a master copy
        dict(name="adamw 8bit", op="adamw", sizes="head", n=4, r=8, d=4096, V=32000, param=BF16, master=False, bits=8, clip=0.0),
    ]


def _log(rng, lo, hi):
    n = int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))
    return n - (n == 3 << 10)


def _width(rng):
    """A row width: often one that the head takes, else any number, odd ones among them."""
    return rng.choice([64, 256, 512, 1024, 2048, 4096]) if rng.random() < 0.5 else _log(rng, 64, 4096)


def draw(rng):
    op = rng.choice(["embed_fwd", "embed_bwd", "norm_fwd", "norm_bwd", "adamw", "adamw"])
    if op == "embed_fwd":
        return dict(op=op, T=_log(rng, 1, 32768), d=_width(rng), V=_log(rng, 100, 128256),
                    scale=rng.choice([1.0, 0.5, 45.25]), out=rng.choice([BF16, F32]), pad=rng.choice([0.0, 0.1]))
    if op == "embed_bwd":
        return dict(op=op, T=_log(rng, 1, 32768), d=_width(rng), V=_log(rng, 100, 128256), scale=rng.choice([1.0, 0.5, 45.25]),
                    dy=rng.choice([BF16, F32]), accumulate=rng.random() < 0.5, pad=rng.choice([0.0, 0.1]))
    if op in ("norm_fwd", "norm_bwd"):
        return dict(op=op, N=_log(rng, 1, 16384), d=_width(rng), stream=rng.choice([BF16, F32]),
                    gate=rng.choice(["none", "row", "channel"]), post=rng.random() < 0.7, fused=rng.random() < 0.5,
                    res_scale=rng.choice([1.0, 0.5]))
    bits = rng.choice([32, 8])
    param = rng.choice([BF16, F32])
    how = dict(param=param, master=param == BF16 and rng.random() < 0.5, bits=bits, clip=1.0 if bits == 32 and rng.random() < 0.7 else 0.0)
    if rng.random() < 0.5:
        return dict(op="adamw", sizes="ragged", count=rng.randint(1, 120), largest=_log(rng, 100, 1000000), **how)
    return dict(op="adamw", sizes="head", n=rng.randint(1, 4), r=rng.randint(1, 8), d=64 * _log(rng, 1, 32), V=_log(rng, 100, 64000), **how)


def _sizes(case):
    """Element counts of the tensors of an optimiser case."""
    if case["sizes"] == "head":
        d = case["d"]
        return [case["n"] * case["r"] * d * d, case["V"] * d, case["r"] * d]
    r = random.Random(case["count"] * 1000003 + case["largest"])
    return [max(1, int(math.exp(r.uniform(0.0, math.log(case["largest"]))))) for _ in range(case["count"])]


def _starts(sizes):
    """Offsets of the tensors in their flat buffers (every tensor starts a block), and the length of a buffer."""
    at, total = [], 0
    for n in sizes:
        at.append(total)
        total += (n + BLOCK - 1) // BLOCK * BLOCK
    return at, total


# ------------------------------------------------------------------------------------------------ inputs

def _tokens(gen, T, V, pad):
    """Zipf-distributed ids (exponent 1.1, id = rank), a share `pad` of them -1 as in a padded batch."""
    p = torch.arange(1, V + 1, dtype=torch.float64, device="cuda").pow(-1.1)
    cdf = torch.cumsum(p / p.sum(), 0)
    x = torch.searchsorted(cdf, torch.rand(T, generator=gen, dtype=torch.float64, device="cuda")).clamp_(max=V - 1).to(torch.int32)
    if pad > 0:
        x = torch.where(torch.rand(T, generator=gen, device="cuda") < pad, torch.full_like(x, -1), x)
    return x


def prepare(case, seed):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(int(seed) * 2654435761 % (1 << 62))

    def randn(*shape, std=1.0, dtype=torch.bfloat16):
        return torch.randn(*shape, generator=gen, device="cuda").mul_(std).to(dtype)

    op = case["op"]
    s = dict(case=case)
    if op == "embed_fwd":
        s["E"] = randn(case["V"], case["d"], std=0.02)
        s["x"] = _tokens(gen, case["T"], case["V"], case["pad"])
    elif op == "embed_bwd":
        s["dy"] = randn(case["T"], case["d"], std=1e-3, dtype=DTYPE[case["dy"]])
        s["x"] = _tokens(gen, case["T"], case["V"], case["pad"])
        s["dE"] = randn(case["V"], case["d"], std=1e-3) if case["accumulate"] else torch.empty(case["V"], case["d"], dtype=torch.bfloat16, device="cuda")
    elif op in ("norm_fwd", "norm_bwd"):
        N, d = case["N"], case["d"]
        # a few channels of a residual stream are much larger than the others
        s["x"] = (torch.randn(N, d, generator=gen, device="cuda") * (1 + 9 * (torch.rand(d, generator=gen, device="cuda") < 0.01))).to(DTYPE[case["stream"]])
        if case["gate"] == "channel" and case["fused"]:
            both = randn(N, 2 * d)
            s["block"], s["gate"] = both[:, :d], both[:, d:]
        else:
            s["block"] = randn(N, d, std=0.5)
            s["gate"] = {"none": lambda: None, "row": lambda: randn(N), "channel": lambda: randn(N, d)}[case["gate"]]()
        s["w_post"] = (1 + torch.randn(d, generator=gen, device="cuda") * 0.1).to(torch.bfloat16) if case["post"] else None
        s["w_pre"] = (1 + torch.randn(d, generator=gen, device="cuda") * 0.1).to(torch.bfloat16)
        if op == "norm_bwd":
            # what the forward pass left behind, and the gradients that come back from above
            x_out, _, s["rstd_post"], s["rstd_pre"] = _norm_fwd(s)
            s["x_out"] = x_out
            del s["x"]
            s["dy"] = randn(N, d, std=1e-3)
            s["dx_out"] = randn(N, d, std=1e-3, dtype=DTYPE[case["stream"]])
    else:
        sizes = _sizes(case)
        at, total = _starts(sizes)
        own_place = torch.zeros(total, dtype=torch.bool, device="cuda")
        for o, n in zip(at, sizes):
            own_place[o:o + n] = True
        # gradients vary in size from row to row; the moments are those of a run under way
        row = torch.randn(total // BLOCK, 1, generator=gen, device="cuda").exp_().mul_(1e-3)
        g = torch.randn(total // BLOCK, BLOCK, generator=gen, device="cuda").mul_(row).view(-1).mul_(own_place)
        m = torch.randn(total // BLOCK, BLOCK, generator=gen, device="cuda").mul_(row * 0.3).view(-1).mul_(own_place)
        v = torch.rand(total // BLOCK, BLOCK, generator=gen, device="cuda").add_(0.5).mul_(row * row).view(-1).mul_(own_place)
        p = torch.randn(total, generator=gen, device="cuda").mul_(0.02).mul_(own_place)
        s["g"] = g.to(DTYPE[case["param"]])
        s["p"] = p.to(DTYPE[case["param"]])
        s["master"] = p if case["master"] else None
        if case["bits"] == 8:
            s["m"], s["m_exp"] = _encode(m, 20, 1 << 19, True)
            s["v"], s["v_exp"] = _encode(v, 19, 1 << 18, False)
        else:
            s["m"], s["v"], s["m_exp"], s["v_exp"] = m, v, None, None
        s["coef"] = torch.full((1,), 0.5, device="cuda") if case["clip"] == 0 else None
        s["hyper"] = dict(lr=3e-4, betas=(0.9, 0.95), eps=1e-8, weight_decay=0.1)
        s["step"], s["seed"] = 100 + int(seed) % 1000, int(seed) % (1 << 31)
        if own:
            from paper_2410_17765_b200 import binding

            def parts(flat, unit=1):
                return None if flat is None else [flat[o // unit:(o + n + unit - 1) // unit] for o, n in zip(at, sizes)]

            # the handle that a training loop keeps
            s["grads"] = parts(s["g"])
            s["optimizer"] = binding.AdamW(parts(s["p"]), bits=case["bits"], master=parts(s["master"]), state=dict(
                m=parts(s["m"]), v=parts(s["v"]), m_exp=parts(s["m_exp"], BLOCK), v_exp=parts(s["v_exp"], BLOCK)))
            s["workspace"] = binding.alloc_workspace(binding.grad_norm_workspace_bytes(s["grads"]))
    return s


# ------------------------------------------------------------------------------------------------ plain forms

def _embed_fwd(s):
    c, x = s["case"], s["x"].long()
    out = s["E"][x.clamp(min=0)].float() * c["scale"]
    return (out * (x >= 0).unsqueeze(1)).to(DTYPE[c["out"]])


def _embed_bwd(s):
    c, x, dE = s["case"], s["x"].long(), s["dE"]
    total = dE.float() if c["accumulate"] else torch.zeros(c["V"], c["d"], device="cuda")
    total.index_add_(0, x.clamp(min=0), s["dy"].float() * (c["scale"] * (x >= 0).float().unsqueeze(1)))
    return dE.copy_(total)


EPS = 1e-6


def _gate(s):
    if s["gate"] is None:
        return 1.0
    g = torch.sigmoid(s["gate"].float())
    return g.unsqueeze(1) if g.dim() == 1 else g


def _norm_fwd(s):
    b = s["block"].float()
    rb = torch.rsqrt(b.square().mean(1) + EPS) if s["w_post"] is not None else None
    u = b if rb is None else b * rb.unsqueeze(1) * s["w_post"].float()
    x = s["case"]["res_scale"] * s["x"].float() + _gate(s) * u
    rx = torch.rsqrt(x.square().mean(1) + EPS)
    return x.to(s["x"].dtype), (x * rx.unsqueeze(1) * s["w_pre"].float()).to(torch.bfloat16), rb, rx


def _norm_bwd(s):
    dy, b, g = s["dy"].float(), s["block"].float(), _gate(s)
    xh = s["x_out"].float() * s["rstd_pre"].unsqueeze(1)
    wdy = dy * s["w_pre"].float()
    t = s["dx_out"].float() + s["rstd_pre"].unsqueeze(1) * (wdy - xh * (wdy * xh).mean(1, keepdim=True))
    r = dict(dx=(s["case"]["res_scale"] * t).to(s["x_out"].dtype), dw_pre=(dy * xh).sum(0).to(torch.bfloat16))
    du, u = g * t, b
    if s["w_post"] is not None:
        bh = b * s["rstd_post"].unsqueeze(1)
        w = s["w_post"].float()
        u = bh * w
        r["dw_post"] = (du * bh).sum(0).to(torch.bfloat16)
        r["dblock"] = (s["rstd_post"].unsqueeze(1) * (w * du - bh * (w * du * bh).mean(1, keepdim=True))).to(torch.bfloat16)
    else:
        r["dblock"] = du.to(torch.bfloat16)
    if s["gate"] is not None:
        dg = t * u * g * (1 - g)
        r["dgate"] = (dg.sum(1) if s["gate"].dim() == 1 else dg).to(torch.bfloat16)
    return r


def _noise(n, seed, step):
    """32 random bits for every element: an integer hash (lowbias32) of its place, keyed by the seed and the step."""
    def mix(x):
        x = x ^ (x >> 16)
        x = (x * 0x7FEB352D) & 0xFFFFFFFF
        x = x ^ (x >> 15)
        x = (x * 0x846CA68B) & 0xFFFFFFFF
        return x ^ (x >> 16)

    one = torch.tensor([seed & 0xFFFFFFFF], device="cuda", dtype=torch.int64)
    key = mix(mix(one) ^ (step & 0xFFFFFFFF))
    i = torch.arange(n, device="cuda", dtype=torch.int64)
    return mix((i & 0xFFFFFFFF) ^ key ^ ((i >> 32) * 0x9E3779B9 & 0xFFFFFFFF))


def _pow2(e):
    """2^(e - 127) for exponent fields e in [0, 254], as fp32 (e = 0: 2^-127)."""
    bits = torch.where(e > 0, e.to(torch.int32) << 23, torch.full_like(e, 1 << 22, dtype=torch.int32))
    return bits.view(torch.float32)


TINY, HUGE = 2.0 ** -112, 2.0 ** 112      # between exponent field 127 and 15


def _encode(x, drop, noise, signed):
    """(codes, exponents) of an 8-bit state: 4 exponent bits and the leading mantissa bits of |x| relative to its
    block's exponent, with `noise` added below the last kept bit."""
    a = x.abs().view(-1, BLOCK)
    e = (a.amax(1, keepdim=True).view(torch.int32) + (1 << drop)) >> 23
    small = (a * _pow2(254 - e)) * TINY
    code = (small.view(torch.int32) + (noise.view(-1, BLOCK) if torch.is_tensor(noise) else noise)) >> drop
    code = torch.where(e > 0, code, torch.zeros_like(code))
    if signed:
        code = torch.where(x.view(-1, BLOCK) < 0, code | 128, code)
    return code.to(torch.uint8).view(-1), e.to(torch.uint8).view(-1)


def _decode(code, e, drop, signed):
    c = code.view(-1, BLOCK).to(torch.int32)
    x = ((((c & 127) if signed else c) << drop).view(torch.float32) * HUGE) * _pow2(e.view(-1, 1))
    return (torch.where(c > 127, -x, x) if signed else x).view(-1)


def _adamw(s):
    c, h, t = s["case"], s["hyper"], s["step"]
    (b1, b2), lr = h["betas"], h["lr"]
    r = {}
    coef = s["coef"]
    g = s["g"].float()
    if c["clip"] > 0:
        r["norm"] = g.square().sum().sqrt().view(1)
        coef = (c["clip"] / (r["norm"] + 1e-6)).clamp(max=1.0)
    g = g * coef
    low = c["bits"] == 8
    m = _decode(s["m"], s["m_exp"], 20, True) if low else s["m"]
    v = _decode(s["v"], s["v_exp"], 19, False) if low else s["v"]
    m = m * b1 + g * (1 - b1)
    v = v * b2 + (g * (1 - b2)) * g
    p = s["p"].float() if s["master"] is None else s["master"]
    p = p * (1 - lr * h["weight_decay"]) - (m * (lr / (1 - b1 ** t))) / (v.sqrt() * (1 / math.sqrt(1 - b2 ** t)) + h["eps"])
    noise = None
    if low or (c["param"] == BF16 and not c["master"]):
        noise = _noise(p.numel(), s["seed"], t)
    if low:
        s["v"], s["v_exp"] = _encode(v, 19, (noise >> 13).to(torch.int32), False)
        # where the second moment rounds to zero so does the first
        code, s["m_exp"] = _encode(m, 20, ((noise & 0xFFFF) << 4).to(torch.int32), True)
        s["m"] = torch.where(s["v"] == 0, torch.zeros_like(code), code)
        r["m"] = _decode(s["m"], s["m_exp"], 20, True).to(torch.bfloat16)      # 8-bit values are exact in bf16
        r["v"] = _decode(s["v"], s["v_exp"], 19, False).to(torch.bfloat16)
    else:
        r["m"], r["v"] = s["m"].copy_(m), s["v"].copy_(v)
    if c["master"]:
        r["master"] = s["master"].copy_(p)
    elif c["param"] == BF16:
        # stochastic rounding: without a master copy nearest rounding would lose every step below half a unit
        p = ((p.view(torch.int32) + ((noise >> 8) & 0xFFFF).to(torch.int32)) & -65536).view(torch.float32)
    r["p"] = s["p"].copy_(p)
    return r


# ------------------------------------------------------------------------------------------------ one pass

def run(s):
    c = s["case"]
    op = c["op"]
    if not own:
        if op == "embed_fwd":
            return _embed_fwd(s)
        if op == "embed_bwd":
            return _embed_bwd(s)
        if op == "norm_fwd":
            x_out, y, rb, rx = _norm_fwd(s)
            return dict(x_out=x_out, y=y, rstd_post=rb, rstd_pre=rx)
        return _norm_bwd(s) if op == "norm_bwd" else _adamw(s)
    from paper_2410_17765_b200 import binding

    if op == "embed_fwd":
        return binding.embed_forward(s["E"], s["x"], scale=c["scale"], out_dtype=DTYPE[c["out"]])
    if op == "embed_bwd":
        return binding.embed_backward(s["dy"], s["x"], c["V"], scale=c["scale"], out=s["dE"], accumulate=c["accumulate"])
    if op == "norm_fwd":
        r = binding.norm_forward(s["x"], s["w_pre"], block=s["block"], gate=s["gate"], w_post=s["w_post"], res_scale=c["res_scale"], eps=EPS)
        return dict(x_out=r["x_out"], y=r["y"], rstd_post=r["rstd_post"], rstd_pre=r["rstd_pre"])
    if op == "norm_bwd":
        r = binding.norm_backward(s["dy"], s["x_out"], s["w_pre"], s["rstd_pre"], dx_out=s["dx_out"], block=s["block"], gate=s["gate"],
                                  w_post=s["w_post"], rstd_post=s["rstd_post"], res_scale=c["res_scale"])
        return {k: v for k, v in r.items() if v is not None}
    r, coef = {}, s["coef"]
    if c["clip"] > 0:
        clip = binding.grad_norm(s["grads"], max_norm=c["clip"], workspace=s["workspace"])
        r["norm"], coef = clip["norm"], clip["coef"]
    s["optimizer"].step(s["grads"], s["step"], coef=coef, seed=s["seed"], **s["hyper"])
    if c["bits"] == 8:
        r["m"] = binding.adamw_state_values(s["m"], s["m_exp"], second=False)
        r["v"] = binding.adamw_state_values(s["v"], s["v_exp"], second=True)
    else:
        r["m"], r["v"] = s["m"], s["v"]
    if c["master"]:
        r["master"] = s["master"]
    r["p"] = s["p"]
    return r


# ------------------------------------------------------------------------------------------------ what a pass cannot do without

def _zipf_distinct(T, V):
    """Expected number of distinct tokens among T."""
    p = torch.arange(1, V + 1, dtype=torch.float64).pow(-1.1)
    return float((1 - (1 - p / p.sum()).pow(T)).sum())


def work(case):
    op = case["op"]
    if op in ("embed_fwd", "embed_bwd"):
        T, d, V = case["T"], case["d"], case["V"]
        rows = _zipf_distinct(T * (1 - case["pad"]), V)
        if op == "embed_fwd":
            return dict(bytes=4 * T + 2 * rows * d + T * d * DTYPE[case["out"]].itemsize, flops=T * d)
        table = 4 * rows * d if case["accumulate"] else 2 * V * d
        return dict(bytes=4 * T + T * (1 - case["pad"]) * d * DTYPE[case["dy"]].itemsize + table, flops=2 * T * d)
    if op in ("norm_fwd", "norm_bwd"):
        N, d = case["N"], case["d"]
        st = DTYPE[case["stream"]].itemsize
        gate = {"none": 0, "row": 2 * N, "channel": 2 * N * d}[case["gate"]]
        weights = 2 * d * (2 if case["post"] else 1)
        stats = 4 * N * (2 if case["post"] else 1)
        if op == "norm_fwd":      # x, block, gate in; x_out, y out
            return dict(bytes=N * d * (2 * st + 4) + gate + weights + stats, flops=12 * N * d)
        return dict(bytes=N * d * (3 * st + 6) + 2 * gate + 2 * weights + stats, flops=30 * N * d)   # dy, x_out, dx_out, block, gate; dx, dblock, dgate
    P = sum(_sizes(case))
    w = DTYPE[case["param"]].itemsize
    per = w + (w + 8 if case["master"] else 2 * w) + (16 if case["bits"] == 32 else 4)
    if case["clip"] > 0:
        per += w        # the norm of all gradients has to be known before the first update
    if case["bits"] == 8:
        per += 6        # the states' values are returned: codes read, bf16 written
    return dict(bytes=P * per, flops=16 * P)


# ------------------------------------------------------------------------------------------------ 64 bits

def exact(case, seed):
    s = prepare(case, seed)
    op = case["op"]
    if op == "embed_fwd":
        x = s["x"].long()
        out = torch.zeros(case["T"], case["d"], dtype=torch.float64, device="cuda")
        keep = torch.nonzero(x != -1).view(-1)
        out[keep] = torch.index_select(s["E"], 0, x[keep]).double() * case["scale"]
        return out
    if op == "embed_bwd":
        # sums of equal tokens as differences of a running sum over the tokens in sorted order
        order = torch.argsort(s["x"], stable=True)
        order = order[s["x"][order] >= 0]
        ids, counts = torch.unique_consecutive(s["x"][order].long(), return_counts=True)
        out = s["dE"].double() if case["accumulate"] else torch.zeros(case["V"], case["d"], dtype=torch.float64, device="cuda")
        if ids.numel():
            running = s["dy"][order].double().cumsum(0)
            last = running[counts.cumsum(0) - 1]
            out[ids] += case["scale"] * torch.cat([last[:1], last[1:] - last[:-1]])
        return out
    if op in ("norm_fwd", "norm_bwd"):
        return _exact_norm(s)
    return _exact_adamw(s)


def _exact_norm(s):
    """The forward pass from its definition; the backward pass as its derivative, by automatic differentiation."""
    c, D = s["case"], torch.float64
    N, d = c["N"], c["d"]
    b, w_pre = s["block"].to(D).requires_grad_(), s["w_pre"].to(D).requires_grad_()
    w_post = s["w_post"].to(D).requires_grad_() if c["post"] else None
    gate = s["gate"].to(D).requires_grad_() if s["gate"] is not None else None

    def rms(z):
        return torch.linalg.vector_norm(z, dim=1).square().div(d).add(EPS).pow(-0.5)

    rb = rms(b) if c["post"] else None
    u = torch.einsum("ij,i,j->ij", b, rb, w_post) if c["post"] else b * 1.0
    if gate is not None:
        g = 1 / (1 + torch.exp(-gate))
        u = torch.einsum("ij,i->ij", u, g) if gate.dim() == 1 else u * g
    if c["op"] == "norm_fwd":
        x = s["x"].to(D) * c["res_scale"] + u
        rx = rms(x)
        y = torch.einsum("ij,i,j->ij", x, rx, w_pre)
        return dict(x_out=x.detach(), y=y.detach(), rstd_post=None if rb is None else rb.detach(), rstd_pre=rx.detach())
    # x_out as it was stored is where the second norm is taken; the residual input reaches it through res_scale
    x_in = torch.zeros(N, d, dtype=D, device="cuda", requires_grad=True)
    x = s["x_out"].to(D) + (c["res_scale"] * x_in + u - u.detach())
    y = torch.einsum("ij,i,j->ij", x, rms(x), w_pre)
    loss = (y * s["dy"].to(D)).sum() + (x * s["dx_out"].to(D)).sum()
    wanted = dict(dx=x_in, dw_pre=w_pre, dblock=b)
    if w_post is not None:
        wanted["dw_post"] = w_post
    if gate is not None:
        wanted["dgate"] = gate
    return dict(zip(wanted, torch.autograd.grad(loss, list(wanted.values()))))


def _exact_adamw(s):
    """Element by element in 64 bits, a slice of the flat buffers at a time (whole blocks)."""
    c, h, t, D = s["case"], s["hyper"], s["step"], torch.float64
    (b1, b2), n = h["betas"], s["p"].numel()
    low = c["bits"] == 8
    r, coef = {}, s["coef"]
    piece = 1 << 26
    if c["clip"] > 0:
        total = sum(float(s["g"][i:i + piece].to(D).pow(2).sum()) for i in range(0, n, piece))
        r["norm"] = torch.tensor([math.sqrt(total)], dtype=D, device="cuda")
        coef = min(1.0, c["clip"] / (math.sqrt(total) + 1e-6))
    else:
        coef = float(coef)
    noise = _noise(n, s["seed"], t) if low or (c["param"] == BF16 and not c["master"]) else None

    def levels(mantissa_bits):
        """Magnitudes of the codes of a 4-bit exponent with this many mantissa bits, in units of the block's exponent."""
        one = 1 << mantissa_bits
        k = torch.arange(16 * one, device="cuda")
        e, f = k // one, (k % one).to(D)
        return torch.where(e > 0, (1 + f / one) * torch.pow(2.0, (e - 15).to(D)), f / one * 2.0 ** -14)

    def values(code, e, bits):
        mag = levels(bits)[(code % 128 if bits == 3 else code).long()]
        x = mag.view(-1, BLOCK) * torch.pow(2.0, e.to(D) - 127).unsqueeze(1)
        return (x * (1 - 2 * (code.view(-1, BLOCK) > 127).to(D)) if bits == 3 else x).view(-1)

    def rounded(x, bits, u):
        """To a neighbouring level, upwards with the probability that keeps the mean: u in [0, 1) decides."""
        a, table = x.abs().view(-1, BLOCK), levels(bits)
        top = a.amax(1, keepdim=True)
        m, e = torch.frexp(top)                                     # top = m 2^e, m in [0.5, 1)
        e = e - 1 + (2 * m >= 2 - 2.0 ** -bits).to(e.dtype)         # room for one step up
        live = (top > 0) & (e + 127 > 0)
        scale = torch.pow(2.0, e.to(D))
        z = a / scale
        lo = (torch.searchsorted(table, z, right=True) - 1).clamp(max=table.numel() - 2)
        part = (z - table[lo]) / (table[lo + 1] - table[lo])
        code = lo + (part + u.view(-1, BLOCK) >= 1).to(lo.dtype)
        out = table[code] * scale * live
        return (out * torch.where(x.view(-1, BLOCK) < 0, -1.0, 1.0)).view(-1)

    outs = dict(p=[], m=[], v=[])
    for i in range(0, n, piece):
        at, blocks = slice(i, min(n, i + piece)), slice(i // BLOCK, min(n, i + piece) // BLOCK)
        g = s["g"][at].to(D) * coef
        m = values(s["m"][at], s["m_exp"][blocks], 3) if low else s["m"][at].to(D)
        v = values(s["v"][at], s["v_exp"][blocks], 4) if low else s["v"][at].to(D)
        m, v = b1 * m + (1 - b1) * g, b2 * v + (1 - b2) * g ** 2
        p = (s["p"] if s["master"] is None else s["master"])[at].to(D)
        p = p - h["lr"] * (h["weight_decay"] * p + (m / (1 - b1 ** t)) / (torch.sqrt(v / (1 - b2 ** t)) + h["eps"]))
        if low:
            v = rounded(v, 4, (noise[at] >> 13).to(D) / (1 << 19))
            m = rounded(m, 3, (noise[at] & 0xFFFF).to(D) / (1 << 16)) * (v > 0)
        outs["p"].append(p)
        outs["m"].append(m)
        outs["v"].append(v)
    r.update({k: torch.cat(x) for k, x in outs.items()})
    if c["master"]:
        r["master"] = r["p"]
    return r
