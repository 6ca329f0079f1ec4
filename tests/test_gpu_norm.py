"""Norms with gate and residual addition against the fp64 restatement.

Bounds, per element: sums over a row or over the rows are fp32 in a tree or in short runs, the exponential of the gate
is good to about 1e-6, so 2e-5 times the sum of the terms' magnitudes covers everything but the last rounding, which is
2^-8 of the value for bf16 and 2^-24 for fp32."""
import numpy as np
import pytest
import torch

from oracle import train_ops as T

pytestmark = pytest.mark.gpu

EPS = 1e-5


def make(N, d, stream, gate, post, fused, seed=0):
    g = torch.Generator().manual_seed(seed)
    v = dict(x=torch.randn(N, d, generator=g).to(stream).cuda(), w_pre=(1 + 0.2 * torch.randn(d, generator=g)).to(torch.bfloat16).cuda())
    both = torch.randn(N, 2 * d, generator=g).to(torch.bfloat16).cuda()
    v["block"] = both[:, :d] if fused else both[:, :d].contiguous()
    v["gate"] = {"none": None, "row": both[:, d].contiguous(), "row strided": both[:, d],
                 "channel": both[:, d:] if fused else both[:, d:].contiguous()}[gate]
    v["w_post"] = (1 + 0.2 * torch.randn(d, generator=g)).to(torch.bfloat16).cuda() if post else None
    v["dy"] = torch.randn(N, d, generator=g).to(torch.bfloat16).cuda()
    v["dx_out"] = torch.randn(N, d, generator=g).to(stream).cuda()
    return v


def f64(t):
    return None if t is None else t.double().cpu().numpy()


def last_rounding(dtype):
    return 2.0 ** -8 if dtype == torch.bfloat16 else 2.0 ** -23


def check_forward(r, v, rs, stream):
    want = T.norm_forward(f64(v["x"]), f64(v["w_pre"]), f64(v["block"]), f64(v["gate"]), f64(v["w_post"]), rs, EPS)
    for k in ("rstd_post", "rstd_pre"):
        if want[k] is not None:
            assert (np.abs(f64(r[k]) - want[k]) <= 1e-5 * want[k]).all()
    parts = np.abs(rs * f64(v["x"]))
    if v["block"] is not None:
        parts = parts + np.abs(want["x_out"] - rs * f64(v["x"]))
        err = np.abs(f64(r["x_out"]) - want["x_out"])
        assert (err <= 2e-5 * parts + last_rounding(stream) * np.abs(want["x_out"])).all(), err.max()
    if want["y"] is not None:
        mag = parts * want["rstd_pre"][:, None] * np.abs(f64(v["w_pre"]))
        err = np.abs(f64(r["y"]) - want["y"])
        assert (err <= 4e-5 * mag + 2.0 ** -8 * np.abs(want["y"])).all(), err.max()


def check_backward(r, v, f, rs, base=None):
    want = T.norm_backward(f64(v["dy"]), f64(f["x_out"]), f64(v["w_pre"]), f64(f["rstd_pre"]), f64(v["dx_out"]), f64(v["block"]),
                           f64(v["gate"]), f64(v["w_post"]), f64(f["rstd_post"]), rs)
    for k, m in want["mag"].items():
        ref = want[k] + (0 if base is None or k not in base else f64(base[k]))
        err = np.abs(f64(r[k]) - ref)
        assert (err <= 2e-5 * m + last_rounding(r[k].dtype) * np.abs(ref) + 1e-37).all(), (k, err.max())
    return want


CASES = [(N, d, stream, gate, post, fused)
         for N, d in [(1, 1), (1, 64), (3, 7), (2, 8), (17, 256), (5, 257), (40, 264), (33, 1000), (9, 1023), (300, 512), (21, 2048), (160, 4096),
                      (7, 4104), (3, 8192), (4, 8191)]
         for stream in (torch.bfloat16, torch.float32)
         for gate, post, fused in [("channel", True, True), ("row", True, False), ("none", False, False), ("row strided", False, True),
                                   ("channel", False, False)]]


@pytest.mark.parametrize("N,d,stream,gate,post,fused", CASES)
def test_forward_and_backward(N, d, stream, gate, post, fused):
    from paper_2410_17765_b200 import binding

    v = make(N, d, stream, gate, post, fused)
    rs = float(np.float32(0.75))
    f = binding.norm_forward(v["x"], v["w_pre"], block=v["block"], gate=v["gate"], w_post=v["w_post"], res_scale=rs, eps=EPS)
    check_forward(f, v, rs, stream)
    kw = dict(dx_out=v["dx_out"], block=v["block"], gate=v["gate"], w_post=v["w_post"], rstd_post=f["rstd_post"], res_scale=rs, eps=EPS)
    r = binding.norm_backward(v["dy"], f["x_out"], v["w_pre"], f["rstd_pre"], **kw)
    check_backward(r, v, f, rs)
    again = binding.norm_backward(v["dy"], f["x_out"], v["w_pre"], f["rstd_pre"], **kw)
    assert all(torch.equal(r[k], again[k]) for k in r if r[k] is not None)


@pytest.mark.parametrize("stream", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("N,d", [(1, 64), (70, 513), (400, 1024)])
def test_norm_alone_and_addition_alone(N, d, stream):
    from paper_2410_17765_b200 import binding

    v = make(N, d, stream, "channel", True, False)
    first = dict(v, block=None, gate=None, w_post=None)
    f = binding.norm_forward(v["x"], v["w_pre"], eps=EPS)
    assert f["x_out"] is v["x"] and f["rstd_post"] is None
    check_forward(f, first, 1.0, stream)
    r = binding.norm_backward(v["dy"], f["x_out"], v["w_pre"], f["rstd_pre"], dx_out=v["dx_out"], eps=EPS)
    check_backward(r, first, f, 1.0)
    assert r["dblock"] is None and r["dgate"] is None and r["dw_post"] is None
    r = binding.norm_backward(v["dy"], f["x_out"], v["w_pre"], f["rstd_pre"], eps=EPS)       # the last norm: nothing else uses x
    check_backward(r, dict(first, dx_out=None), f, 1.0)
    last = dict(v, w_pre=None, dy=None)
    f = binding.norm_forward(v["x"], block=v["block"], gate=v["gate"], w_post=v["w_post"], eps=EPS)
    assert f["y"] is None
    check_forward(f, last, 1.0, stream)
    r = binding.norm_backward(None, f["x_out"], dx_out=v["dx_out"], block=v["block"], gate=v["gate"], w_post=v["w_post"],
                              rstd_post=f["rstd_post"], eps=EPS)
    check_backward(r, last, f, 1.0)
    assert r["dw_pre"] is None


def test_gradient_against_differences():
    """The kernel's gradients along random directions against differences of the fp64 forward pass: 2^-8 of rounding per
    element averages out over thousands, 1 % holds with margin."""
    from paper_2410_17765_b200 import binding

    v = make(64, 384, torch.float32, "channel", True, True, seed=4)
    f = binding.norm_forward(v["x"], v["w_pre"], block=v["block"], gate=v["gate"], w_post=v["w_post"], res_scale=0.5, eps=EPS)
    r = binding.norm_backward(v["dy"], f["x_out"], v["w_pre"], f["rstd_pre"], dx_out=v["dx_out"], block=v["block"], gate=v["gate"],
                              w_post=v["w_post"], rstd_post=f["rstd_post"], res_scale=0.5, eps=EPS)
    a = {k: f64(v[k]) for k in ("x", "w_pre", "block", "gate", "w_post")}
    dy, dx_out = f64(v["dy"]), f64(v["dx_out"])

    def loss(a):
        o = T.norm_forward(a["x"], a["w_pre"], a["block"], a["gate"], a["w_post"], 0.5, EPS)
        return np.sum(o["y"] * dy) + np.sum(o["x_out"] * dx_out)

    for key, name in dict(x="dx", block="dblock", gate="dgate", w_pre="dw_pre", w_post="dw_post").items():
        got = f64(r[name])
        direction = got / np.linalg.norm(got)
        h = 1e-4
        diff = (loss({**a, key: a[key] + h * direction}) - loss({**a, key: a[key] - h * direction})) / (2 * h)
        assert abs(diff - np.linalg.norm(got)) <= 1e-2 * abs(diff), name


def test_in_place_addition_accumulated_weights_and_skipped_outputs():
    from paper_2410_17765_b200 import binding

    v = make(50, 640, torch.bfloat16, "channel", True, True)
    kw = dict(block=v["block"], gate=v["gate"], w_post=v["w_post"], eps=EPS)
    f = binding.norm_forward(v["x"], v["w_pre"], **kw)
    x = v["x"].clone()
    g = binding.norm_forward(x, v["w_pre"], out={"x_out": x}, **kw)
    assert g["x_out"] is x and torch.equal(x, f["x_out"]) and torch.equal(g["y"], f["y"])
    kw.update(dx_out=v["dx_out"], rstd_post=f["rstd_post"])
    r = binding.norm_backward(v["dy"], f["x_out"], v["w_pre"], f["rstd_pre"], **kw)
    both = torch.empty(50, 1280, dtype=torch.bfloat16, device="cuda")
    base = {k: torch.randn(640, device="cuda").to(torch.bfloat16) for k in ("dw_pre", "dw_post")}
    out = {"dx": v["dx_out"].clone(), "dblock": both[:, :640], "dgate": both[:, 640:], **{k: b.clone() for k, b in base.items()}}
    kw["dx_out"] = out["dx"]                              # the gradient of the stream in place
    a = binding.norm_backward(v["dy"], f["x_out"], v["w_pre"], f["rstd_pre"], out=out, accumulate=True, **kw)
    for k in ("dx", "dblock", "dgate"):
        assert torch.equal(a[k], r[k])
    check_backward(a, v, f, 1.0, base)
    kw["dx_out"] = v["dx_out"]
    s = binding.norm_backward(v["dy"], f["x_out"], v["w_pre"], f["rstd_pre"], skip=("dx", "dw_pre", "dw_post"), **kw)
    assert s["dx"] is None and s["dw_pre"] is None and torch.equal(s["dblock"], r["dblock"]) and torch.equal(s["dgate"], r["dgate"])
    s = binding.norm_backward(v["dy"], f["x_out"], v["w_pre"], f["rstd_pre"], skip=("dx", "dblock", "dgate", "dw_post"), **kw)
    assert torch.equal(s["dw_pre"], r["dw_pre"])


@pytest.mark.parametrize("d", [96, 97])
def test_rows_of_zeros_extreme_gates_and_non_finite_rows(d):
    from paper_2410_17765_b200 import binding

    v = make(40, d, torch.float32, "channel", True, False)
    v["block"][3] = 0
    v["x"][3] = 0                                          # a row of nothing: y = 0, rstd = eps^-1/2
    v["gate"][4] = -float("inf")
    v["gate"][5] = float("inf")
    v["gate"][6] = torch.finfo(torch.bfloat16).min
    v["gate"][7] = torch.finfo(torch.bfloat16).max
    f = binding.norm_forward(v["x"], v["w_pre"], block=v["block"], gate=v["gate"], w_post=v["w_post"], eps=EPS)
    check_forward(f, v, 1.0, torch.float32)
    assert not f["y"][3].any() and torch.equal(f["x_out"][4], v["x"][4]) and torch.equal(f["x_out"][6], v["x"][6])
    kw = dict(dx_out=v["dx_out"], block=v["block"], gate=v["gate"], w_post=v["w_post"], rstd_post=f["rstd_post"], eps=EPS)
    r = binding.norm_backward(v["dy"], f["x_out"], v["w_pre"], f["rstd_pre"], **kw)
    check_backward(r, v, f, 1.0)
    assert not r["dgate"][4:8].any() and not r["dblock"][4].any()
    x = v["x"].clone()
    x[9], x[11, 2] = float("nan"), float("inf")
    g = binding.norm_forward(x, v["w_pre"], block=v["block"], gate=v["gate"], w_post=v["w_post"], eps=EPS)
    rest = [i for i in range(40) if i not in (9, 11)]
    assert torch.isnan(g["y"][9]).all() and torch.equal(g["y"][rest], f["y"][rest]) and torch.equal(g["x_out"][rest], f["x_out"][rest])
    b = binding.norm_backward(v["dy"], g["x_out"], v["w_pre"], g["rstd_pre"], **kw)
    assert torch.equal(b["dx"][rest], r["dx"][rest]) and torch.equal(b["dblock"][rest], r["dblock"][rest])


def test_no_rows():
    from paper_2410_17765_b200 import binding

    x = torch.empty(0, 64, dtype=torch.bfloat16, device="cuda")
    w = torch.ones(64, dtype=torch.bfloat16, device="cuda")
    f = binding.norm_forward(x, w, block=x, w_post=w)
    r = binding.norm_backward(x, f["x_out"], w, f["rstd_pre"], block=x, w_post=w, rstd_post=f["rstd_post"],
                              out={"dw_pre": w.clone(), "dw_post": w.clone()})
    assert not r["dw_pre"].any() and not r["dw_post"].any() and r["dx"].shape == (0, 64)


def test_another_stream():
    from paper_2410_17765_b200 import binding

    v = make(2000, 1024, torch.bfloat16, "channel", True, True)
    kw = dict(block=v["block"], gate=v["gate"], w_post=v["w_post"], eps=EPS)
    want = binding.norm_forward(v["x"], v["w_pre"], **kw)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        got = binding.norm_forward(v["x"], v["w_pre"], **kw)
        back = binding.norm_backward(v["dy"], got["x_out"], v["w_pre"], got["rstd_pre"], dx_out=v["dx_out"], rstd_post=got["rstd_post"], **kw)
    side.synchronize()
    assert torch.equal(got["y"], want["y"])
    check_backward(back, v, want, 1.0)


def test_offsets_beyond_32_bits():
    from paper_2410_17765_b200 import binding

    N, d = 530000, 4096                                    # 2.2e9 elements
    x = torch.ones(N, d, dtype=torch.bfloat16, device="cuda")
    x[-1] = 3.0
    w = torch.full((d,), 2.0, dtype=torch.bfloat16, device="cuda")
    f = binding.norm_forward(x, w, eps=1e-12)
    assert (f["y"][-1] == 2).all() and (f["y"][-2] == 2).all() and (f["y"][0] == 2).all()
    assert abs(float(f["rstd_pre"][-1]) - 1 / 3) < 1e-6
    r = binding.norm_backward(f["y"], x, w, f["rstd_pre"], dx_out=x, out={"dx": x}, eps=1e-12)
    # w dy = 4 and xh = 1 everywhere: the projection takes all of it away and dx is dx_out
    assert (r["dx"][-1] == 3).all() and (r["dx"][-2] == 1).all()
    assert torch.allclose(r["dw_pre"].float(), torch.full((d,), 2.0 * N, device="cuda"), rtol=2.0 ** -8)


def test_refusals():
    from paper_2410_17765_b200 import binding

    v = make(4, 32, torch.bfloat16, "channel", True, False)
    x, w, b, g, p = v["x"], v["w_pre"], v["block"], v["gate"], v["w_post"]
    f = binding.norm_forward(x, w, block=b, gate=g, w_post=p)
    bad = [lambda: binding.norm_forward(x), lambda: binding.norm_forward(x.half(), w), lambda: binding.norm_forward(x, w.float()),
           lambda: binding.norm_forward(x, w[:31]), lambda: binding.norm_forward(x, w, gate=g), lambda: binding.norm_forward(x, w, w_post=p),
           lambda: binding.norm_forward(x, w, res_scale=0.5), lambda: binding.norm_forward(x, w, block=b[:3]),
           lambda: binding.norm_forward(x, w, block=b.float()), lambda: binding.norm_forward(x, w, block=b, gate=g[:, :31]),
           lambda: binding.norm_forward(x, w, eps=0.0), lambda: binding.norm_forward(x, w, eps=float("nan")),
           lambda: binding.norm_forward(x, w, block=b, res_scale=float("inf")), lambda: binding.norm_forward(x.cpu(), w.cpu()),
           lambda: binding.norm_forward(x, w.cpu()), lambda: binding.norm_forward(x.t(), w),
           lambda: binding.norm_forward(x[:1].expand(4, 32), w), lambda: binding.norm_forward(x, w, block=b, out={"x_out": x[:2]}),
           lambda: binding.norm_forward(torch.ones(1, 8193, dtype=torch.bfloat16, device="cuda"), torch.ones(8193, dtype=torch.bfloat16, device="cuda")),
           lambda: binding.norm_backward(None, x, w, f["rstd_pre"]), lambda: binding.norm_backward(v["dy"], x, w),
           lambda: binding.norm_backward(v["dy"].float(), x, w, f["rstd_pre"]),
           lambda: binding.norm_backward(v["dy"], x, w, f["rstd_pre"], block=b, w_post=p),
           lambda: binding.norm_backward(v["dy"], x, w, f["rstd_pre"], accumulate=True),
           lambda: binding.norm_backward(v["dy"], x, w, f["rstd_pre"], skip=("dx", "dw_pre")),
           lambda: binding.norm_backward(v["dy"], x, w, f["rstd_pre"], workspace=torch.empty(256, dtype=torch.uint8, device="cuda"))]
    for i, c in enumerate(bad):
        with pytest.raises(binding.CpmtpError):
            c()
            pytest.fail(f"refusal {i} did not happen")
