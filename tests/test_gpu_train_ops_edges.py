"""Edges of the training-step operators' range of numbers, against the fp64 restatement."""
import numpy as np
import pytest
import torch

from oracle import train_ops as T

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("eps", [0.0, 1e-30, 1e-22, 1e-12])
@pytest.mark.parametrize("n,offset", [(1024, 0), (1024 + 100, 0), (1024, 1)])
@pytest.mark.parametrize("bits", [32, 8])
def test_second_moments_below_the_normal_numbers(bits, n, offset, eps):
    """With an eps that does not hide them, roots of subnormal second moments make the step: in whole blocks, in a tensor's last one
    and in tensors that allow no wide accesses alike.  The moments are compared as fp32 defines them, the update of
    a parameter is good to 1e-6 of it and 4 * 2^-24 of the parameter."""
    from paper_2410_17765_b200 import binding

    rng = np.random.default_rng(n + offset)
    betas, lr, wd = (0.9, 0.99), 0.01, 0.1
    f = np.float32
    p = torch.zeros(n + offset, device="cuda")[offset:]
    p.copy_(torch.from_numpy(rng.normal(size=n).astype(f)))
    dtype, blocks = (torch.float32, n) if bits == 32 else (torch.uint8, -(-n // 256))
    state = {k: [torch.zeros(n + offset, dtype=dtype, device="cuda")[offset:]] for k in ("m", "v")}
    if bits == 8:
        state.update({k: [torch.zeros(blocks, dtype=torch.uint8, device="cuda")] for k in ("m_exp", "v_exp")})
    opt = binding.AdamW([p], bits=bits, state=state)
    m, v = np.zeros(n, f), np.zeros(n, f)
    for t in range(1, 4):
        # moments from 2.5e-43 up (178 units of the smallest number), every third one a normal number
        size = np.where(np.arange(n) % 3 == 2, 1e-17, 1e-20)
        g = (size * rng.uniform(0.5, 2, n) * rng.choice([-1, 1], n)).astype(f)
        before = p.cpu().numpy().astype(np.float64)
        m0, v0 = m, v
        m1 = m0 * f(betas[0]) + g * f(1 - betas[0])
        v1 = v0 * f(betas[1]) + (g * f(1 - betas[1])) * g
        assert (v1 > 2e-43).all() and (v1 < 2.0 ** -126).any()
        opt.step([torch.cat([torch.zeros(offset), torch.from_numpy(g)]).cuda()[offset:]], t, lr=lr, betas=betas, eps=eps, weight_decay=wd, seed=5)
        upd = (m1.astype(np.float64) / (1 - betas[0] ** t)) / (np.sqrt(v1.astype(np.float64) / (1 - betas[1] ** t)) + eps)
        want = before - lr * (wd * before + upd)
        err = np.abs(p.cpu().numpy() - want)
        assert (err <= 1e-6 * np.abs(lr * upd) + 4 * 2.0 ** -24 * np.maximum(np.abs(want), np.abs(before))).all(), (t, err.max())
        if bits == 32:
            m, v = opt.m[0].cpu().numpy(), opt.v[0].cpu().numpy()
        else:
            m, v = (T.decode(getattr(opt, k)[0].cpu().numpy(), getattr(opt, k + "_exp")[0].cpu().numpy(), k == "v") for k in ("m", "v"))
