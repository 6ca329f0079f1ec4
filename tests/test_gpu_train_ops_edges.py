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


@pytest.mark.parametrize("gate", ["row", "channel"])
@pytest.mark.parametrize("stream", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("d", [64, 100, 1024, 1027, 4096, 4352, 4354])
@pytest.mark.parametrize("whole", [True, False])
def test_gradients_of_open_and_closed_gates(gate, stream, d, whole):
    """g (1 - g) keeps its digits wherever it is a number at all; bounds as in the tests of the norms: 2e-5 of the terms' magnitudes, which hold the
    factor g (1 - g), and half a unit of the output."""
    from paper_2410_17765_b200 import binding

    logits = np.array([0, 3, 6, 9, 10, 11, 12, 14, 16, 17, 20, 30, 50, 80, -10, -12, -16, -17, -30, -80], np.float32)
    N = 40
    gen = torch.Generator().manual_seed(d)

    def draw(*shape, dtype=torch.bfloat16):
        return torch.randn(*shape, generator=gen).to(dtype).cuda()

    x, block, dy, dx_out = draw(N, d, dtype=stream), draw(N, d), draw(N, d), draw(N, d, dtype=stream)
    w_pre, w_post = draw(d), draw(d)
    at = np.arange(N) if gate == "row" else np.arange(N)[:, None] + np.arange(d)[None]
    z = torch.from_numpy(logits[at % logits.size]).to(torch.bfloat16).cuda()
    f = binding.norm_forward(x, w_pre, block=block, gate=z, w_post=w_post)
    # with all outputs, and with the gate's gradient alone (another form of the kernel)
    r = binding.norm_backward(dy, f["x_out"], w_pre, f["rstd_pre"], dx_out=dx_out, block=block, gate=z, w_post=w_post, rstd_post=f["rstd_post"],
                              skip=() if whole else ("dx", "dblock", "dw_post", "dw_pre"))
    a = [t.double().cpu().numpy() for t in (dy, f["x_out"], w_pre, f["rstd_pre"], dx_out, block, z, w_post, f["rstd_post"])]
    want = T.norm_backward(*a)
    for k in [k for k in want["mag"] if r[k] is not None]:
        last = 2.0 ** -8 if r[k].dtype == torch.bfloat16 else 2.0 ** -23
        err = np.abs(r[k].double().cpu().numpy() - want[k])
        assert (err <= 2e-5 * want["mag"][k] + last * np.abs(want[k]) + 1e-37).all(), (k, err.max())
    assert r["dgate"] is not None


@pytest.mark.parametrize("gate", ["none", "row", "channel"])
@pytest.mark.parametrize("d", [64, 100, 4096, 4352])
def test_rows_of_zeros_with_the_smallest_eps(gate, d):
    """rstd is then 2^63; the gradients of rows of zeros are finite and those of the others do not notice."""
    from paper_2410_17765_b200 import binding

    eps, N = 2.0 ** -126, 24
    gen = torch.Generator().manual_seed(d)

    def draw(*shape):
        return torch.randn(*shape, generator=gen).to(torch.bfloat16).cuda()

    def check(r, *a):
        want = T.norm_backward(*[None if t is None else t.double().cpu().numpy() for t in a])
        for k in want["mag"]:
            err = np.abs(r[k].double().cpu().numpy() - want[k])
            assert (err <= 2e-5 * want["mag"][k] + 2.0 ** -8 * np.abs(want[k]) + 1e-37).all(), (k, err.max())

    x, block, dy, dx_out, w_pre, w_post = draw(N, d), draw(N, d), draw(N, d), draw(N, d), draw(d), draw(d)
    z = {"none": None, "row": draw(N), "channel": draw(N, d)}[gate]
    block[::3] = 0
    f = binding.norm_forward(x, w_pre, block=block, gate=z, w_post=w_post, eps=eps)
    assert float(f["rstd_post"][0]) == 2.0 ** 63
    r = binding.norm_backward(dy, f["x_out"], w_pre, f["rstd_pre"], dx_out=dx_out, block=block, gate=z, w_post=w_post, rstd_post=f["rstd_post"], eps=eps)
    check(r, dy, f["x_out"], w_pre, f["rstd_pre"], dx_out, block, z, w_post, f["rstd_post"])
    x[::2] = 0
    f = binding.norm_forward(x, w_pre, eps=eps)
    assert float(f["rstd_pre"][0]) == 2.0 ** 63 and not f["y"][0].any()
    check(binding.norm_backward(dy, x, w_pre, f["rstd_pre"], dx_out=dx_out, eps=eps), dy, x, w_pre, f["rstd_pre"], dx_out)
    with pytest.raises(binding.CpmtpError):
        binding.norm_forward(x, w_pre, eps=1e-40)
