"""The operators together, as a training step uses them."""
import math

import numpy as np
import pytest
import torch

from oracle import cp_head
from oracle import train_ops as T

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("bits,master", [(8, False), (32, True)])
def test_the_loss_falls(bits, master):
    from paper_2410_17765_b200 import train_demo

    losses = train_demo.train(60, bits=bits, master=master)
    n, V = 3, 1024
    assert abs(losses[0] - n * math.log(V)) < 1.0           # an untrained head is close to uniform
    # the walk follows its rule nine times out of ten: most of the way from uniform to that is learnt in 60 steps
    assert losses[-1] < 0.6 * losses[0]
    assert all(math.isfinite(x) for x in losses)
    assert train_demo.train(5, bits=bits, master=master) == losses[:5]       # bit-reproducible


def test_gradients_of_the_whole_step_against_differences():
    """Along the gradient, the fp64 loss of the whole model changes by what the kernels' gradient says: bf16 roundings of
    intermediate results (2^-9 each, a handful one after the other) leave a few per cent at these small sizes at most."""
    from paper_2410_17765_b200 import train_demo

    cfg = train_demo.Config(batch=4, length=14, d=64, V=300, n=2, r=2, aux_coef=0.05)
    m = train_demo.Model(cfg, seed=3)
    tokens = train_demo.walk(cfg, torch.Generator(device="cuda").manual_seed(5))
    f = m.forward(tokens)
    g = m.backward(f)
    assert int(m.status.item()) == 0
    x, targets = f["cur"].cpu().numpy(), f["targets"].cpu()
    params = {k: getattr(m, k).double().cpu().numpy() for k in m.names}

    def loss(p):
        x0 = T.embed_forward(p["E"], x, math.sqrt(cfg.d))
        y0 = T.norm_forward(x0, p["w_in"])["y"]
        both = y0 @ p["W_block"].T
        h = T.norm_forward(x0, p["w_pre"], both[:, :cfg.d], both[:, cfg.d:], p["w_post"])["y"]
        args = [torch.from_numpy(a) for a in (h, p["W_head"], p["E"], p["W_g"])]
        return cp_head.forward(*args, targets, cfg.n, cfg.r, aux_coef=cfg.aux_coef).loss

    assert abs(loss(params) - float(f["loss"])) < 2e-2
    for k in m.names:
        got = g[k].double().cpu().numpy()
        size = np.linalg.norm(got)
        h = 1e-3 / max(1.0, np.abs(got / size).max())
        diff = (loss({**params, k: params[k] + h * got / size}) - loss({**params, k: params[k] - h * got / size})) / (2 * h)
        assert abs(diff - size) < 0.05 * size, (k, diff, size)


def test_a_step_replays_from_a_cuda_graph():
    from paper_2410_17765_b200 import binding, train_demo

    cfg = train_demo.Config(batch=4, length=20, d=128, V=512, n=2, r=2)
    gen = torch.Generator(device="cuda").manual_seed(9)
    tokens = train_demo.walk(cfg, gen)
    models = [train_demo.Model(cfg, seed=1) for _ in range(2)]
    graph, side = torch.cuda.CUDAGraph(), torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        train_demo.Model(cfg, seed=1).step(tokens, 1, lr=1e-3)               # first launches outside the capture
    side.synchronize()
    with torch.cuda.graph(graph, stream=side):
        out = models[0].step(tokens, 1, lr=1e-3)
    for _ in range(3):
        graph.replay()
        want = models[1].step(tokens, 1, lr=1e-3)
        torch.cuda.synchronize()
        assert torch.equal(out["loss"], want["loss"]) and torch.equal(out["norm"], want["norm"])
        for k in models[0].names:
            assert torch.equal(getattr(models[0], k), getattr(models[1], k)), k
    assert binding.load_library().cpmtp_version() >= 130
