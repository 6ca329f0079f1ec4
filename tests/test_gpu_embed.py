"""Embedding lookup and its gradient against the fp64 restatement.

Bounds, per element: the lookup is one fp32 product and one rounding (bf16: 2^-8 of the value, fp32: 2^-23); the gradient
is a sum of c fp32 terms in some order, (c + 2) 2^-24 times the sum of their magnitudes, and one rounding to bf16."""
import numpy as np
import pytest
import torch

from oracle import train_ops as T

pytestmark = pytest.mark.gpu


def tokens(rng, n, V, pad=0.0):
    x = np.minimum(rng.zipf(1.3, n) - 1, V - 1).astype(np.int32)
    x[rng.random(n) < pad] = -1
    return x


def bf16(a):
    return torch.from_numpy(np.asarray(a, np.float32)).to(torch.bfloat16).cuda()


def check_grad(got, dy, x, V, scale, base=None):
    want, mag, terms = T.embed_backward(dy.float().cpu().numpy(), x, V, scale, None if base is None else base.float().cpu().numpy())
    err = np.abs(got.float().cpu().numpy() - want)
    assert (err <= (terms[:, None] + 2) * 2.0 ** -24 * mag + 2.0 ** -8 * np.abs(want) + 1e-37).all(), err.max()


SHAPES = [(1, 1, 1), (1, 5, 64), (2, 3, 8), (31, 2, 7), (32, 40, 256), (33, 40, 264), (97, 1000, 255), (1000, 50, 257), (4097, 700, 40),
          (2049, 300000, 16), (300, 517, 1000), (65, 9, 4096)]


@pytest.mark.parametrize("n,V,d", SHAPES)
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_lookup(n, V, d, dtype):
    from paper_2410_17765_b200 import binding

    rng = np.random.default_rng(n + d)
    E, x = bf16(rng.normal(size=(V, d))), tokens(rng, n, V, 0.1)
    st = torch.zeros(1, dtype=torch.int32, device="cuda")
    out = binding.embed_forward(E, torch.from_numpy(x).cuda(), scale=1.7, out_dtype=dtype, dev_status=st)
    want = T.embed_forward(E.float().cpu().numpy(), x, np.float32(1.7))
    assert out.dtype == dtype and out.shape == (n, d)
    assert (np.abs(out.float().cpu().numpy() - want) <= (2.0 ** -8 if dtype == torch.bfloat16 else 2.0 ** -23) * np.abs(want)).all()
    assert int(st.item()) == 0


@pytest.mark.parametrize("n,V,d", SHAPES)
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("accumulate", [False, True])
def test_gradient(n, V, d, dtype, accumulate):
    from paper_2410_17765_b200 import binding

    rng = np.random.default_rng(n * 7 + d)
    x = tokens(rng, n, V, 0.1)
    dy = torch.from_numpy(rng.normal(size=(n, d)).astype(np.float32)).to(dtype).cuda()
    out = bf16(rng.normal(size=(V, d)))
    base = out.clone() if accumulate else None
    if not accumulate:
        out.fill_(float("nan"))                       # every row has to be written
    got = binding.embed_backward(dy, torch.from_numpy(x).cuda(), V, scale=0.6, out=out, accumulate=accumulate)
    assert got is out
    check_grad(got, dy, x, V, float(np.float32(0.6)), base)
    if accumulate:
        rest = np.setdiff1d(np.arange(V), x)
        assert torch.equal(got[rest], base[rest])


@pytest.mark.parametrize("n", [1024, 1025, 8192, 8193, 16385, 33000, 65536, 65537, 150000])
@pytest.mark.parametrize("V", [300, 40000, 262144])
def test_gradient_over_the_ways_to_sort(n, V):
    """One block, a cluster of eight with one to eight keys a thread, several launches; one to three digits."""
    from paper_2410_17765_b200 import binding

    rng = np.random.default_rng(n + V)
    x = tokens(rng, n, V, 0.05)
    dy = bf16(rng.normal(size=(n, 8)))
    got = binding.embed_backward(dy, torch.from_numpy(x).cuda(), V, out=torch.full((V, 8), float("nan"), dtype=torch.bfloat16, device="cuda"))
    check_grad(got, dy, x, V, 1.0)


@pytest.mark.parametrize("kind", ["one token", "all padding", "two interleaved", "sorted", "every row once"])
def test_gradient_of_extreme_token_counts(kind):
    from paper_2410_17765_b200 import binding

    rng = np.random.default_rng(5)
    n, V, d = 5000, 5000, 72
    x = {"one token": np.full(n, 4321), "all padding": np.full(n, -1), "two interleaved": np.arange(n) % 2 * 4999,
         "sorted": np.sort(rng.integers(0, V, n)), "every row once": rng.permutation(V)}[kind].astype(np.int32)
    dy = bf16(rng.normal(size=(n, d)))
    got = binding.embed_backward(dy, torch.from_numpy(x).cuda(), V, out=torch.full((V, d), float("nan"), dtype=torch.bfloat16, device="cuda"))
    check_grad(got, dy, x, V, 1.0)
    again = binding.embed_backward(dy, torch.from_numpy(x).cuda(), V)
    assert torch.equal(got, again)                    # no dependence on the order of arrival


def test_tokens_out_of_range_are_clamped_and_reported():
    from paper_2410_17765_b200 import binding

    rng = np.random.default_rng(6)
    E, x = bf16(rng.normal(size=(10, 16))), np.array([0, -2, 10, -1, 2 ** 31 - 1, -2 ** 31], np.int32)
    st = torch.zeros(1, dtype=torch.int32, device="cuda")
    out = binding.embed_forward(E, torch.from_numpy(x).cuda(), dev_status=st)
    assert int(st.item()) == 1
    assert torch.equal(out, torch.stack([E[0], E[0], E[9], torch.zeros_like(E[0]), E[9], E[0]]))
    st.zero_()
    dy = bf16(rng.normal(size=(6, 16)))
    got = binding.embed_backward(dy, torch.from_numpy(x).cuda(), 10, dev_status=st)
    assert int(st.item()) == 1
    check_grad(got, dy, x, 10, 1.0)


def test_strided_rows_misaligned_tables_and_batched_tokens():
    from paper_2410_17765_b200 import binding

    rng = np.random.default_rng(7)
    V, d, n = 50, 24, 60
    wide = bf16(rng.normal(size=(V, 2 * d + 1)))
    x = torch.from_numpy(tokens(rng, n, V)).cuda()
    for E in (wide[:, :d], wide[:, d + 1:]):          # a row stride of 49 elements; one that starts off a 16-byte boundary
        out = torch.zeros(n, 3 * d, dtype=torch.float32, device="cuda")
        binding.embed_forward(E, x, out=out[:, d:2 * d])
        assert torch.equal(out[:, d:2 * d], E[x.long()].float())
        assert not out[:, :d].any() and not out[:, 2 * d:].any()
    dy = torch.from_numpy(rng.normal(size=(n, 2 * d + 1)).astype(np.float32)).cuda()
    table = torch.full((V, 3 * d), 7.0, dtype=torch.bfloat16, device="cuda")
    binding.embed_backward(dy[:, 1:d + 1], x, V, out=table[:, d:2 * d])
    check_grad(table[:, d:2 * d].contiguous(), dy[:, 1:d + 1], x.cpu().numpy(), V, 1.0)
    assert (table[:, :d] == 7).all() and (table[:, 2 * d:] == 7).all()
    E = wide[:, :d].contiguous()
    assert torch.equal(binding.embed_forward(E, x.view(3, 20)), E[x.long()].view(3, 20, d))
    dy3 = bf16(rng.normal(size=(3, 20, d)))
    check_grad(binding.embed_backward(dy3, x.view(3, 20), V), dy3.view(n, d), x.cpu().numpy(), V, 1.0)


def test_no_tokens():
    from paper_2410_17765_b200 import binding

    E = bf16(np.ones((5, 16)))
    x = torch.empty(0, dtype=torch.int32, device="cuda")
    assert binding.embed_forward(E, x).shape == (0, 16)
    dy = torch.empty(0, 16, dtype=torch.bfloat16, device="cuda")
    assert not binding.embed_backward(dy, x, 5, out=torch.ones(5, 16, dtype=torch.bfloat16, device="cuda")).any()
    kept = torch.ones(5, 16, dtype=torch.bfloat16, device="cuda")
    assert binding.embed_backward(dy, x, 5, out=kept, accumulate=True).all()


def test_offsets_beyond_32_bits():
    from paper_2410_17765_b200 import binding

    V, d = 540000, 4096                               # 2.2e9 elements
    E = torch.zeros(V, d, dtype=torch.bfloat16, device="cuda")
    x = torch.tensor([V - 1, 0, V - 2, V - 1], dtype=torch.int32, device="cuda")
    E[x.long()] = bf16(np.random.default_rng(8).normal(size=(4, d)))
    assert torch.equal(binding.embed_forward(E, x), E[x.long()])
    dy = bf16(np.random.default_rng(9).normal(size=(4, d)))
    got = binding.embed_backward(dy, x, V, out=E)
    want = torch.stack([(dy[0].float() + dy[3].float()).to(torch.bfloat16), dy[1], dy[2]])
    assert torch.equal(got[[V - 1, 0, V - 2]], want)
    assert not got[1:V - 2].any()


def test_non_finite_rows_stay_in_their_rows():
    from paper_2410_17765_b200 import binding

    dy = torch.ones(40, 32, dtype=torch.bfloat16, device="cuda")
    dy[3], dy[5] = float("inf"), float("nan")
    x = torch.arange(40, dtype=torch.int32, device="cuda") % 8
    x[4] = -1
    dy[4] = float("nan")                              # padding: never looked at
    got = binding.embed_backward(dy, x, 8)
    assert torch.isinf(got[3]).all() and torch.isnan(got[5]).all()
    assert torch.isfinite(got[[0, 1, 2, 4, 6, 7]]).all() and (got[4] == 4).all()


def test_tied_table_gets_both_gradients():
    """The head's dE, then the lookup's added to it: one rounding more than the sum of the two in fp64."""
    from paper_2410_17765_b200 import binding, synth

    s = synth.CONFIGS["tiny"]
    inp = synth.make_inputs(s, seed=3)
    dev = [t.cuda() for t in (inp.h, inp.W_head, inp.E, inp.W_g, inp.x)]
    saved = binding.Saved.alloc(binding.make_shape(s.N, s.d, s.V, s.n, s.r))
    binding.forward(*dev, saved=saved)
    g = binding.backward(*dev, saved)
    head = g["dE"].clone()
    x = inp.x[:, 0].contiguous().cuda()
    binding.embed_backward(g["dh"], x, s.V, scale=2.0, out=g["dE"], accumulate=True)
    check_grad(g["dE"], g["dh"], x.cpu().numpy(), s.V, 2.0, head)


def test_refusals():
    from paper_2410_17765_b200 import binding

    E = bf16(np.ones((5, 16)))
    x = torch.zeros(4, dtype=torch.int32, device="cuda")
    dy = bf16(np.ones((4, 16)))
    bad = [lambda: binding.embed_forward(E.float(), x), lambda: binding.embed_forward(E, x.long()), lambda: binding.embed_forward(E, x.cpu()),
           lambda: binding.embed_forward(E.cpu(), x.cpu()), lambda: binding.embed_forward(E.t(), x),
           lambda: binding.embed_forward(E, x, out_dtype=torch.float16), lambda: binding.embed_forward(E, x, out=dy[:3]),
           lambda: binding.embed_backward(dy.half(), x, 5), lambda: binding.embed_backward(dy[:3], x, 5),
           lambda: binding.embed_backward(dy, x, 5, accumulate=True), lambda: binding.embed_backward(dy, x, 5, out=E[:4]),
           lambda: binding.embed_backward(dy[:1].expand(4, 16), x, 5), lambda: binding.embed_backward(dy, x, 0),
           lambda: binding.embed_backward(dy, x, 5, workspace=torch.empty(256, dtype=torch.uint8, device="cuda"))]
    for f in bad:
        with pytest.raises(binding.CpmtpError):
            f()
