"""Optimiser steps by a clock on the device: the same bits as steps that the host numbers, one by one and replayed from a graph."""
import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu

HYPER = dict(betas=(0.9, 0.99), eps=1e-8, weight_decay=0.1)
SIZES = [1, 255, 256, 8193, 30011]


def make(bits, param, master, factors=True):
    from paper_2410_17765_b200 import binding

    gen = torch.Generator(device="cuda").manual_seed(8)

    def draw(n):
        return torch.randn(n, generator=gen, device="cuda").to(param)

    params = [draw(n) for n in SIZES]
    kw = dict(lr_scale=[1.0, 0.5, 0.3, 1.0, 0.1], decay_scale=[1.0, 0.0, 0.7, 1.0, 0.3]) if factors else {}
    return binding.AdamW(params, bits=bits, master=master, **kw), [draw(n) * 0.01 for n in SIZES], draw


def same(a, b):
    for i in range(len(a.params)):
        assert torch.equal(a.params[i], b.params[i]), i
        for k in ("m", "v", "m_exp", "v_exp", "master"):
            x, y = getattr(a, k)[i], getattr(b, k)[i]
            assert (x is None and y is None) or torch.equal(x, y), (i, k)


FORMS = [(32, torch.float32, False), (32, torch.bfloat16, True), (32, torch.bfloat16, False), (8, torch.bfloat16, False), (8, torch.bfloat16, True),
         (8, torch.float32, False)]


@pytest.mark.parametrize("bits,param,master", FORMS)
def test_replays_are_the_steps_that_follow(bits, param, master):
    """Bit for bit, with gradients, learning rate and clipping that change from step to step."""
    from paper_2410_17765_b200 import binding

    a, grads, draw = make(bits, param, master)
    b, _, _ = make(bits, param, master)
    clock = binding.StepClock(0.01, seed=77)
    coef = torch.ones(1, device="cuda")
    graph, side = torch.cuda.CUDAGraph(), torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        w, _, _ = make(bits, param, master)
        w.step(grads, binding.StepClock(0.01), coef=coef, **HYPER)           # first launches outside the capture
    side.synchronize()
    with torch.cuda.graph(graph, stream=side):
        a.step(grads, clock, coef=coef, **HYPER)
    assert int(clock.step) == 0                                              # (captured, not run)
    for t in range(1, 31):
        lr = 0.01 * min(1.0, t / 5)
        for g in grads:
            g.copy_(draw(g.numel()) * 0.01)
        coef.fill_(1.0 / t)
        clock.lr.fill_(lr)
        graph.replay()
        b.step(grads, t, lr=lr, coef=coef, seed=77, **HYPER)
        same(a, b)
        assert int(clock.step) == t


def test_a_clock_starts_where_it_is_set():
    from paper_2410_17765_b200 import binding

    for start in (0, 1, 999, 123456, (1 << 32) - 2):
        a, grads, _ = make(8, torch.bfloat16, False)
        b, _, _ = make(8, torch.bfloat16, False)
        clock = binding.StepClock(1e-3, step=start, seed=(1 << 32) + 5)
        for t in range(start + 1, start + 4):
            a.step(grads, clock, **HYPER)
            b.step(grads, t, lr=1e-3, seed=(1 << 32) + 5, **HYPER)
            same(a, b)
        clock.step.fill_(6)                                                  # a restored run
        a.step(grads, clock, **HYPER)
        b.step(grads, 7, lr=1e-3, seed=5, **HYPER)
        same(a, b)


def test_more_tensors_than_one_launch_holds():
    from paper_2410_17765_b200 import binding

    gen = torch.Generator(device="cuda").manual_seed(1)
    params = [torch.randn(37 * i % 700 + 1, generator=gen, device="cuda").to(torch.bfloat16) for i in range(650)]
    grads = [p * 0.01 for p in params]
    a, b = binding.AdamW([p.clone() for p in params], bits=8), binding.AdamW([p.clone() for p in params], bits=8)
    clock = binding.StepClock(0.01)
    for t in range(1, 4):
        a.step(grads, clock)
        b.step(grads, t, lr=0.01)
    same(a, b)
    assert int(clock.step) == 3


def test_a_skipped_step_advances_the_clock():
    from paper_2410_17765_b200 import binding

    a, grads, _ = make(8, torch.bfloat16, False)
    before = [p.clone() for p in a.params]
    clock = binding.StepClock(0.01)
    a.step(grads, clock, coef=torch.full((1,), float("nan"), device="cuda"))
    assert int(clock.step) == 1 and all(torch.equal(x, y) for x, y in zip(a.params, before))


def test_noise_of_replays_keeps_the_mean():
    """Steps of a hundredth of a bf16 unit, replayed: with one step's noise every time, a hundredth of the elements would move by a
    unit a step and the others never."""
    from paper_2410_17765_b200 import binding

    n, steps, lr = 1 << 16, 50, 2.0 ** -8 / 100                              # below 1 a unit is 2^-8
    p, g = torch.ones(n, dtype=torch.bfloat16, device="cuda"), torch.ones(n, dtype=torch.bfloat16, device="cuda")
    opt, clock = binding.AdamW([p]), binding.StepClock(lr)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        binding.AdamW([p.clone()]).step([g], binding.StepClock(lr), weight_decay=0.0)
    side.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        opt.step([g], clock, weight_decay=0.0)
    for _ in range(steps):
        graph.replay()
    x = 1 - p.double()
    # each step is a coin of variance unit^2 * 0.01 per element: five standard errors of the mean over n
    assert abs(float(x.mean()) - steps * lr) < 5 * 2.0 ** -8 * np.sqrt(steps * 0.01 / n) + 1e-6
    # and the coins are thrown anew: about 1 - 0.99^50 = 0.395 of the elements have moved
    assert abs(float((x > 0).double().mean()) - 0.395) < 0.01


@pytest.mark.parametrize("bits,master", [(8, False), (32, True)])
def test_a_captured_training_step_trains(bits, master):
    """A step of the demo's whole model, replayed, against eager steps with the same numbers."""
    from paper_2410_17765_b200 import binding, train_demo

    cfg = train_demo.Config(batch=4, length=20, d=128, V=512, n=2, r=2)
    gen = torch.Generator(device="cuda").manual_seed(9)
    batches = [train_demo.walk(cfg, gen) for _ in range(12)]
    a, b = (train_demo.Model(cfg, seed=1, bits=bits, master=master) for _ in range(2))
    tokens, clock = batches[0].clone(), binding.StepClock(1e-3, seed=3)
    graph, side = torch.cuda.CUDAGraph(), torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        train_demo.Model(cfg, seed=1, bits=bits, master=master).step(tokens, binding.StepClock(1e-3))
    side.synchronize()
    with torch.cuda.graph(graph, stream=side):
        out = a.step(tokens, clock)
    for t, batch in enumerate(batches, 1):
        tokens.copy_(batch)
        graph.replay()
        f = b.forward(batch)
        grads = [b.backward(f)[k] for k in b.names]
        b.optimizer.step(grads, t, lr=1e-3, seed=3, coef=binding.grad_norm(grads, max_norm=1.0)["coef"])
        assert torch.equal(out["loss"], f["loss"]), t
        for k in a.names:
            assert torch.equal(getattr(a, k), getattr(b, k)), (t, k)


def test_refusals():
    from paper_2410_17765_b200 import binding

    p = torch.zeros(64, device="cuda")
    opt, clock = binding.AdamW([p]), binding.StepClock(0.1)
    wrong = binding.StepClock(0.1)
    wrong.block = wrong.block[:8]
    bad = [lambda: opt.step([p], clock, lr=0.1), lambda: opt.step([p], clock, seed=3), lambda: opt.step([p], 1),
           lambda: opt.step([p], clock, betas=(1.0, 0.9)), lambda: opt.step([p], clock, eps=-1.0), lambda: opt.step([p], wrong),
           lambda: opt.step([p], binding.StepClock(0.1, device="cpu")), lambda: binding.StepClock(-1.0), lambda: binding.StepClock(float("nan")),
           lambda: binding.StepClock(0.1, step=-1)]
    for i, f in enumerate(bad):
        with pytest.raises(binding.CpmtpError):
            f()
            pytest.fail(f"refusal {i} did not happen")
    assert int(clock.step) == 0
