"""AdamW over many tensors, 8-bit states and gradient clipping against the fp64 restatement.

Bounds: moments are a few fp32 roundings, 4 * 2^-24 of their terms' magnitudes; the update of a parameter divides with a
few ulps of error, 1e-6 of it, and the parameter itself takes 4 * 2^-24 of its value, plus half a unit where it is
rounded to bf16 (2^-8) or a whole one where it is rounded stochastically (2^-7).  8-bit codes are defined on fp32
operations and have to be equal."""
import numpy as np
import pytest
import torch

from oracle import train_ops as T

pytestmark = pytest.mark.gpu

HYPER = dict(lr=0.01, betas=(0.9, 0.99), eps=1e-8, weight_decay=0.1)
SIZES = [1, 7, 255, 256, 257, 8192, 8193, 30011, 512]


def flat(t):
    return t.detach().float().cpu().numpy().astype(np.float64).ravel()


def make(sizes, param, master, bits, seed=0, grad=None, offset=0):
    from paper_2410_17765_b200 import binding

    g = torch.Generator().manual_seed(seed)

    def draw(n, std, dtype, positive=False):
        a = torch.randn(n + offset, generator=g) * std
        return (a.abs() if positive else a).to(dtype).cuda()[offset:]

    params = [draw(n, 0.5, param) for n in sizes]
    grads = [draw(n, 1e-2, grad or param) for n in sizes]
    masters = [p.float() + 1e-3 * draw(p.numel(), 0.5, torch.float32) if master else None for p in params]
    if bits == 32:
        state = dict(m=[draw(n, 1e-2, torch.float32) for n in sizes], v=[draw(n, 1e-4, torch.float32, True) for n in sizes])
    else:
        state = dict(m=[], v=[], m_exp=[], v_exp=[])
        for n in sizes:
            m, v = draw(n, 1e-2, torch.float32), draw(n, 1e-4, torch.float32, True)
            for k, a in (("m", m), ("v", v)):
                c, e = T.encode(a.cpu().numpy(), np.zeros(n), k == "v")
                codes = torch.zeros(n + offset, dtype=torch.uint8)
                codes[offset:] = torch.from_numpy(c)
                state[k].append(codes.cuda()[offset:])
                state[k + "_exp"].append(torch.from_numpy(e).cuda())
    return params, grads, masters, state, binding


def run_and_check(sizes, param, master, bits, coef=None, steps=2, grad=None, offset=0, seed=11, skip=()):
    params, grads, masters, state, binding = make(sizes, param, master, bits, grad=grad, offset=offset)
    opt = binding.AdamW(params, bits=bits, master=masters if master else False, state=state)
    scale = 1.0 if coef is None else float(coef.item())
    for t in range(5, 5 + steps):
        before = [dict(p=flat(masters[i] if master else p), m=state["m"][i].cpu().numpy().copy(), v=state["v"][i].cpu().numpy().copy(),
                       **({} if bits == 32 else dict(me=state["m_exp"][i].cpu().numpy().copy(), ve=state["v_exp"][i].cpu().numpy().copy())))
                  for i, p in enumerate(params)]
        opt.step([None if i in skip else g for i, g in enumerate(grads)], t, coef=coef, seed=seed, **HYPER)
        place = 0
        for i, (n, b) in enumerate(zip(sizes, before)):
            here, place = place, place + -(-n // 256) * 256
            p_now = flat(masters[i] if master else params[i])
            if i in skip:
                assert (p_now == b["p"]).all() and (state["m"][i].cpu().numpy() == b["m"]).all()
                continue
            if bits == 32:
                m0, v0 = b["m"].astype(np.float64), b["v"].astype(np.float64)
            else:
                m0, v0 = T.decode(b["m"], b["me"], False), T.decode(b["v"], b["ve"], True)
            p, m, v = T.adamw(b["p"], flat(grads[i]), m0, v0, step=t, coef=scale, **HYPER)
            if bits == 32:
                g = np.abs(flat(grads[i]) * scale)
                assert (np.abs(flat(state["m"][i]) - m) <= 4 * 2.0 ** -24 * (np.abs(0.9 * m0) + 0.1 * g)).all()
                assert (np.abs(flat(state["v"][i]) - v) <= 4 * 2.0 ** -24 * (0.99 * v0 + 0.01 * g * g)).all()
            else:
                want = T.adamw_states_8bit(flat(grads[i]), b["m"], b["me"], b["v"], b["ve"], betas=HYPER["betas"], step=t, seed=seed,
                                           coef=scale, place=here)
                for k, w in zip(("m", "m_exp", "v", "v_exp"), want):
                    assert (state[k][i].cpu().numpy() == w).all(), k
            rounding = 0.0 if master or param == torch.float32 else 2.0 ** -7
            bound = (4 * 2.0 ** -24 + rounding) * np.maximum(np.abs(p), np.abs(b["p"])) + 1e-6 * np.abs(p - b["p"] * (1 - HYPER["lr"] * 0.1))
            err = np.abs(p_now - p)
            assert (err <= bound).all(), (i, n, err.max())
            if master:
                assert torch.equal(params[i], masters[i].to(torch.bfloat16))


@pytest.mark.parametrize("param,master", [(torch.bfloat16, True), (torch.bfloat16, False), (torch.float32, False)])
@pytest.mark.parametrize("bits", [32, 8])
@pytest.mark.parametrize("offset", [0, 1])
def test_step(param, master, bits, offset):
    run_and_check(SIZES, param, master, bits, offset=offset)


@pytest.mark.parametrize("scale", [1e-22, 1e-18, 1e-10, 1e6, 1e15])
def test_eight_bit_states_far_from_one(scale):
    """Exponents at which the powers of two of coding and decoding no longer fit into one factor, down to subnormal moments."""
    from paper_2410_17765_b200 import binding

    n = 4096 + 300
    gen = torch.Generator().manual_seed(1)
    p = torch.zeros(n, device="cuda")
    opt = binding.AdamW([p], bits=8)
    m, v = np.zeros(n, np.uint8), np.zeros(n, np.uint8)
    me, ve = np.zeros(-(-n // 256), np.uint8), np.zeros(-(-n // 256), np.uint8)
    for t in range(1, 5):
        g = (torch.randn(n, generator=gen) * scale).cuda()
        g[256:512] = 0                                     # and a block of nothing
        opt.step([g], t, lr=1e-3, betas=HYPER["betas"], seed=3)
        m, me, v, ve = T.adamw_states_8bit(g.cpu().numpy(), m, me, v, ve, betas=HYPER["betas"], step=t, seed=3)
        for name, got, want in (("m", opt.m, m), ("m_exp", opt.m_exp, me), ("v", opt.v, v), ("v_exp", opt.v_exp, ve)):
            assert (got[0].cpu().numpy() == want).all(), (name, t)
    assert torch.isfinite(p).all()


@pytest.mark.parametrize("bits", [32, 8])
def test_mixed_types_and_scaled_gradients(bits):
    run_and_check([1000, 4096], torch.bfloat16, True, bits, grad=torch.float32, coef=torch.full((1,), 0.37, device="cuda"))
    run_and_check([1000, 4096], torch.float32, False, bits, grad=torch.bfloat16, skip=(0,))


@pytest.mark.parametrize("bits", [32, 8])
def test_more_tensors_than_one_launch_holds(bits):
    """Also: the noise of a tensor does not depend on how the tensors are spread over launches."""
    run_and_check([(37 * i) % 700 + 1 for i in range(650)], torch.bfloat16, False, bits, steps=1, skip=(3, 400))


def test_stochastic_rounding_of_parameters_keeps_the_mean():
    """Steps of a hundredth of a bf16 unit: nearest rounding would never move, on average they add up."""
    from paper_2410_17765_b200 import binding

    n = 1 << 16
    p = torch.ones(n, dtype=torch.bfloat16, device="cuda")
    opt = binding.AdamW([p])
    g = torch.ones(n, dtype=torch.bfloat16, device="cuda")
    steps, lr = 50, 2.0 ** -8 / 100                        # below 1 a unit is 2^-8
    for t in range(1, steps + 1):
        opt.step([g], t, lr=lr, weight_decay=0.0, seed=t)
    moved = 1 - float(p.double().mean())                   # a constant gradient moves a parameter by lr a step
    # each step is a coin of variance unit^2 * 0.01 per element: five standard errors of the mean over n
    assert abs(moved - steps * lr) < 5 * 2.0 ** -8 * np.sqrt(steps * 0.01 / n) + 1e-6


def test_per_tensor_factors():
    from paper_2410_17765_b200 import binding

    ps = [torch.ones(300, device="cuda") for _ in range(3)]
    g = [torch.zeros(300, device="cuda"), torch.zeros(300, device="cuda"), torch.ones(300, device="cuda")]
    opt = binding.AdamW(ps, lr_scale=[1.0, 1.0, 0.5], decay_scale=[1.0, 0.0, 0.0])
    opt.step(g, 1, lr=0.1, weight_decay=0.5)
    assert torch.allclose(ps[0], torch.full_like(ps[0], 0.95)) and (ps[1] == 1).all() and torch.allclose(ps[2], torch.full_like(ps[2], 0.95))


@pytest.mark.parametrize("bits", [32, 8])
def test_non_finite_gradients(bits):
    from paper_2410_17765_b200 import binding

    p = torch.ones(1024, device="cuda")
    opt = binding.AdamW([p], bits=bits)
    g = torch.full((1024,), 0.1, device="cuda")
    g[300] = float("nan")
    clip = binding.grad_norm([g], max_norm=1.0)
    assert torch.isnan(clip["norm"]).all() and torch.isnan(clip["coef"]).all()
    opt.step([g], 1, lr=0.1, coef=clip["coef"])            # skipped as a whole
    assert (p == 1).all() and not opt.m[0].any() and not opt.v[0].any()
    opt.step([g], 1, lr=0.1)                               # without the clip it goes where it goes: its own element, and block of states
    assert torch.isnan(p[300]) and torch.isfinite(p[:300]).all() and torch.isfinite(p[301:]).all()
    if bits == 8:
        values = binding.adamw_state_values(opt.m[0], opt.m_exp[0], second=False)
        assert torch.isnan(values[256:512]).all() and torch.isfinite(values[:256]).all() and torch.isfinite(values[512:]).all()
    g[300] = float("inf")
    assert torch.isnan(binding.grad_norm([g])["coef"]).all()


@pytest.mark.parametrize("n", [1, 255, 256, 5000])
@pytest.mark.parametrize("offset", [0, 1])
def test_state_values(n, offset):
    from paper_2410_17765_b200 import binding

    rng = np.random.default_rng(n)
    code, e = rng.integers(0, 256, n + offset).astype(np.uint8), rng.integers(20, 235, -(-n // 256)).astype(np.uint8)
    c = torch.from_numpy(code).cuda()[offset:]
    for second in (False, True):
        got = binding.adamw_state_values(c, torch.from_numpy(e).cuda(), second=second)
        assert (got.float().cpu().numpy() == T.decode(code[offset:], e, second)).all()


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("sizes", [[1], [5, 8192, 1], [100000, 33], [17] * 350])
def test_grad_norm(dtype, sizes):
    from paper_2410_17765_b200 import binding

    g = torch.Generator().manual_seed(len(sizes))
    grads = [torch.randn(n, generator=g).to(dtype).cuda() for n in sizes]
    want = np.sqrt(sum(np.sum(flat(t) ** 2) for t in grads))
    for max_norm in (0.1, 1e9, float("inf")):
        r = binding.grad_norm(grads, max_norm=max_norm)
        # at most 30 squares meet in fp32 per accumulator here, the rest is fp64
        assert abs(float(r["norm"]) - want) <= 3e-6 * want
        assert abs(float(r["coef"]) - min(1.0, max_norm / (want + 1e-6))) <= 4e-6
    zero = [torch.zeros_like(t) for t in grads]
    r = binding.grad_norm(zero, max_norm=1.0)
    assert float(r["norm"]) == 0 and float(r["coef"]) == 1
    again = binding.grad_norm(grads)
    assert torch.equal(again["norm"], binding.grad_norm(grads + [None])["norm"])


def test_more_than_2_to_the_31_elements():
    from paper_2410_17765_b200 import binding

    n = (1 << 31) + 1000
    p = torch.zeros(n, dtype=torch.bfloat16, device="cuda")
    g = torch.zeros(n, dtype=torch.bfloat16, device="cuda")
    g[-700:], g[:5] = 1.0, 1.0
    opt = binding.AdamW([p], bits=8)
    opt.step([g], 1, lr=0.5, weight_decay=0.0, coef=binding.grad_norm([g], max_norm=1e9)["coef"])
    assert torch.allclose(p[-700:].float(), torch.full((700,), -0.5, device="cuda"), rtol=2.0 ** -7) and not p[5:-700].any()
    want, we, vc, ve = T.adamw_states_8bit(np.ones(232), np.zeros(232, np.uint8), np.zeros(1, np.uint8), np.zeros(232, np.uint8),
                                           np.zeros(1, np.uint8), betas=(0.9, 0.95), step=1, seed=0, place=(1 << 31) + 768)
    assert (opt.m[0][-232:].cpu().numpy() == want).all() and (opt.v[0][-232:].cpu().numpy() == vc).all()
    assert abs(float(binding.grad_norm([g])["norm"]) - np.sqrt(705)) < 1e-3


def test_refusals():
    from paper_2410_17765_b200 import binding

    p = torch.zeros(64, dtype=torch.bfloat16, device="cuda")
    g = torch.zeros_like(p)
    opt = binding.AdamW([p])
    step = dict(lr=0.1)
    bad = [lambda: binding.AdamW([p], bits=16), lambda: binding.AdamW([p.half()]), lambda: binding.AdamW([p.cpu()]),
           lambda: binding.AdamW([p.view(8, 8).t()]), lambda: binding.AdamW([p], master=[p]), lambda: binding.AdamW([p], lr_scale=[1.0, 2.0]),
           lambda: binding.AdamW([p], state=dict(m=[p], v=[p])), lambda: binding.AdamW([p.float()], master=[p.float()]),
           lambda: opt.step([], 1, **step), lambda: opt.step([g[:32]], 1, **step), lambda: opt.step([g.cpu()], 1, **step),
           lambda: opt.step([g], 0, **step), lambda: opt.step([g], 1, lr=-1.0), lambda: opt.step([g], 1, lr=float("nan")),
           lambda: opt.step([g], 1, betas=(1.0, 0.9), **step), lambda: opt.step([g], 1, eps=float("inf"), **step),
           lambda: opt.step([g], 1, coef=torch.ones(1), **step), lambda: opt.step([g], 1, coef=torch.ones(1, dtype=torch.float64, device="cuda"), **step),
           lambda: binding.grad_norm([]), lambda: binding.grad_norm([g], max_norm=0.0), lambda: binding.grad_norm([g], max_norm=float("nan")),
           lambda: binding.grad_norm([g.half()]), lambda: binding.grad_norm([g], workspace=torch.empty(8, dtype=torch.uint8, device="cuda")),
           lambda: binding.adamw_state_values(p, p, second=True),
           lambda: binding.adamw_state_values(torch.zeros(257, dtype=torch.uint8, device="cuda"), torch.zeros(1, dtype=torch.uint8, device="cuda"), second=True)]
    for i, c in enumerate(bad):
        with pytest.raises(binding.CpmtpError):
            c()
            pytest.fail(f"refusal {i} did not happen")
    assert not p.any()
