"""Sampling from logits against the fp64 restatement.

Tokens and numbers of kept entries are compared exactly wherever the oracle's decisions lie further than 2^-31 from their borders (its
`gap`, relative to the masses compared; weights are off by 2^-32 at most and summed exactly).  Log-probabilities: 2^-24 of the value for
the rounding and 2^-30 for the sums."""
import numpy as np
import pytest
import torch

from oracle import serve_ops as S

pytestmark = pytest.mark.gpu


def check(logits, uniform, T=1.0, k=0, p=1.0, min_p=0.0, given=None, sure=True, **how):
    from paper_2410_17765_b200 import binding

    N, V = logits.shape
    st = torch.zeros(1, dtype=torch.int32, device="cuda")
    r = binding.sample_logits(logits, uniform, temperature=T, top_k=k, top_p=p, min_p=min_p, given=given, want_kept=True, dev_status=st, **how)
    assert int(st.item()) == 0
    x, u = logits.float().cpu().numpy(), uniform.cpu().numpy().astype(np.float64)

    def rows(v):
        return v.cpu().numpy() if torch.is_tensor(v) else np.full(N, v, np.int64 if isinstance(v, int) else np.float32)

    Ts, ks, ps, ms = rows(T), rows(k), rows(p), rows(min_p)
    tokens, logp, kept = (r[n].cpu().numpy() for n in ("tokens", "logp", "kept"))
    decided = 0
    for i in range(N):
        w = S.sample(x[i], float(np.clip(u[i], 0, 1)), float(Ts[i]), int(ks[i]), float(ps[i]), float(ms[i]))
        if not w["gap"] > 2.0 ** -31:
            continue
        decided += 1
        assert tokens[i] == w["token"] and kept[i] == w["kept"], (i, tokens[i], w["token"], kept[i], w["kept"])
        if np.isneginf(w["logp"]):
            assert np.isneginf(logp[i])
        else:
            assert abs(logp[i] - w["logp"]) <= 2.0 ** -24 * abs(w["logp"]) + 2.0 ** -30
        if given is not None:
            g = int(given[i])
            want = w["all"][g] if 0 <= g < V else -np.inf
            want = want if want > -3.5e38 else -np.inf          # (below the range of fp32, which ends at 3.4e38)
            got = float(r["logp_given"][i])
            assert got == want if np.isneginf(want) else abs(got - want) <= 2.0 ** -24 * abs(want) + 2.0 ** -30
    assert decided == N or not sure
    return r


def draw(N, V, seed, dtype, std=2.5):
    g = torch.Generator(device="cuda").manual_seed(seed)
    return (torch.randn(N, V, generator=g, device="cuda") * std).to(dtype), torch.rand(N, generator=g, device="cuda")


FILTERS = [dict(), dict(k=1), dict(k=50), dict(p=0.9), dict(p=0.5, k=1000), dict(min_p=0.05), dict(k=40, p=0.95, min_p=0.02), dict(T=0.0), dict(T=0.2, p=0.99), dict(T=3.0, p=0.7),
           dict(p=0.0), dict(min_p=2.0), dict(k=10 ** 9)]


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("how", FILTERS, ids=str)
@pytest.mark.parametrize("N,V", [(3, 1), (4, 2), (5, 33), (7, 1000), (3, 4097), (2, 32003), (1, 128256), (1, 300001)])
def test_filters(N, V, how, dtype):
    x, u = draw(N, V, V, dtype)
    given = torch.from_numpy(np.random.default_rng(V).integers(-1, V, N).astype(np.int32)).cuda()
    check(x, u, given=given, sure=False, **how)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_rows_with_settings_of_their_own(dtype):
    N = 64
    x, u = draw(N, 5003, 1, dtype)
    g = torch.Generator(device="cuda").manual_seed(2)
    r = torch.rand(4, N, generator=g, device="cuda")
    check(x, u, T=torch.where(r[0] < 0.2, 0.0, r[0] * 2), k=((r[1] - 0.3) * 100).to(torch.int32), p=r[2] * 1.5, min_p=r[3] * 0.2 - 0.05, sure=False,
          given=x.float().argmax(1).to(torch.int32))


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("how", [dict(), dict(k=7), dict(p=0.3), dict(p=0.77, k=100), dict(min_p=1.0)], ids=str)
def test_equal_logits_go_by_index(how, dtype):
    """Rows of one value, of two and of a few: whole runs of equals at every border."""
    u = torch.tensor([0.1, 0.6, 0.33], device="cuda")
    x = torch.zeros(3, 2500, device="cuda")
    x[1, ::3] = 1.0
    x[2] = torch.arange(2500, device="cuda") % 5
    check(x.to(dtype), u, **how)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_all_uniforms_of_a_small_row(dtype):
    """The whole range of the drawn number: 256 equal steps over four entries of equal weight, and beyond both ends."""
    u = torch.cat([(torch.arange(256, device="cuda") + 0.5) / 256, torch.tensor([0.0, -1.0, 1.0, 5.0], device="cuda")])
    x = torch.full((260, 9), -float("inf"), device="cuda")
    x[:, 1::2] = 0.25
    r = check(x[:256].to(dtype), u[:256])
    assert r["tokens"].tolist() == [1 + 2 * (i // 64) for i in range(256)]
    from paper_2410_17765_b200 import binding

    assert binding.sample_logits(x[256:].to(dtype), u[256:])["tokens"].tolist() == [1, 1, 7, 7]


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_infinities_and_nan(dtype):
    inf, nan = float("inf"), float("nan")
    x = torch.tensor([[nan, -inf, -inf, nan, -inf], [nan, 1.0, -inf, 2.0, 1.0], [inf, 3.0, inf, nan, -inf], [-0.0, 0.0, -0.0, 0.0, nan], [-inf, -3e38, -inf, -3e38, -3e38],
                      [3e38, -3e38, 3e38, 0.0, nan]], device="cuda").to(dtype)
    u = torch.tensor([0.5, 0.5, 0.7, 0.6, 0.5, 0.75], device="cuda")
    given = torch.tensor([1, 2, 0, 1, 3, 1], dtype=torch.int32, device="cuda")
    for how in (dict(), dict(k=2), dict(p=0.6), dict(min_p=0.1), dict(T=0.0), dict(T=1e-30)):
        check(x, u, given=given, sure=False, **how)
        for others in ([2, 4, 1, 4, 1, 3], [3, 3, 4, 2, 0, 4]):
            check(x, u, given=torch.tensor(others, dtype=torch.int32, device="cuda"), sure=False, **how)
    r = check(x[:1], u[:1])
    assert r["tokens"].tolist() == [-1] and r["kept"].tolist() == [0] and r["logp"].tolist() == [-inf]


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("V,ld,shift", [(1001, 1001, 0), (1001, 1011, 3), (4096, 5000, 1), (4096, 4096, 0), (777, 1024, 8)])
def test_strided_rows(V, ld, shift, dtype):
    wide, u = draw(9, ld + 16, 3, dtype)
    flat = wide.view(-1)
    x = torch.as_strided(flat, (9, V), (ld, 1), shift)
    check(x, u, p=0.9, sure=False)


@pytest.mark.parametrize("N", [1, 8, 40, 150, 700])
@pytest.mark.parametrize("how", [dict(k=30, p=0.9), dict(p=0.8), dict(k=1500, min_p=1e-4)], ids=str)
def test_numbers_of_rows(N, how):
    x, u = draw(N, 2049, N, torch.bfloat16)
    check(x, u, sure=False, **how)


def test_many_rows_of_equals():
    """Long runs of equal logits in rows that small blocks take."""
    x = (torch.arange(320 * 3000, device="cuda") % 7).view(320, 3000).float()
    u = torch.rand(320, generator=torch.Generator(device="cuda").manual_seed(1), device="cuda")
    for how in (dict(k=1100), dict(p=0.6), dict(k=2900, p=0.99)):
        check(x, u, sure=False, **how)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("V", [1000, 50001, 128256])
def test_top_p_near_one(V, dtype):
    """Borders with little mass behind them, and with little before them."""
    x, u = draw(20, V, V, dtype)
    near = [1 - 2.0 ** -k for k in range(4, 20)] + [2.0 ** -k for k in (3, 7, 11, 20)]
    for min_p in (0.0, 1e-4):
        check(x, u, p=torch.tensor(near, dtype=torch.float32, device="cuda"), min_p=min_p, given=x.argmax(1).int(), sure=False)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("N,V", [(5, 128256), (5, 20011), (300, 20011), (5, 700)])
def test_top_k_wherever_the_largest_lie(N, V, dtype):
    """In order, in one thread's pieces, in few values, at the ends: the borders that a part of the row gives are too low then, or too long runs lie above them."""
    g = torch.Generator(device="cuda").manual_seed(V)
    x, u = draw(5, V, N, torch.float32)
    at = torch.arange(V, device="cuda")
    x[0] = x[0].sort().values
    x[1] = x[1].sort(descending=True).values
    x[2] += 20.0 * ((at // 8) % 256 == 5)
    x[3] = torch.randint(0, 3, (V,), generator=g, device="cuda").float() * (at < V - 3) + 5.0 * (at >= V - 2)
    x[4, V // 2:] = float("-inf")
    x, u = x.repeat(N // 5, 1).to(dtype), torch.rand(N, generator=g, device="cuda")
    for k in (2, 50, 224, 225, 448, 449, 2048):
        check(x, u, k=k, p=0.9 if k % 2 == 0 else 1.0, given=x.argmin(1).int(), sure=False)


def test_peaked_and_flat_rows():
    x, u = draw(6, 50000, 8, torch.float32, std=1e-3)
    check(x, u, p=0.8, sure=False)
    x[:, 123] = 80.0
    check(x, u, p=0.8)
    check(x, u)


@pytest.mark.parametrize("how", [dict(p=0.9), dict(k=30), dict(k=5000, p=0.7), dict(min_p=0.01)], ids=str)
def test_results_do_not_depend_on_the_batch(how):
    """Rows alone, in a few and in many: shared out over 8, 4, 2 and 1 blocks."""
    from paper_2410_17765_b200 import binding

    names = dict(p="top_p", k="top_k", min_p="min_p")
    x, u = draw(400, 50000, 12, torch.float32)
    args = {names[k]: v for k, v in how.items()}
    want = binding.sample_logits(x, u, want_kept=True, **args)
    for n in (1, 3, 20, 60, 140, 200):
        got = binding.sample_logits(x[:n], u[:n], want_kept=True, **args)
        assert all(torch.equal(got[k], want[k][:n]) for k in want)


@pytest.mark.parametrize("how", [dict(p=0.9), dict(k=100000, p=0.8), dict(min_p=0.5), dict()], ids=str)
def test_a_vocabulary_of_millions(how):
    x, u = draw(1, 3000001, 5, torch.float32)
    check(x, u, sure=False, **how)


def test_shares_of_draws():
    """20000 draws of one row: each count within five standard deviations of its mean."""
    from paper_2410_17765_b200 import binding

    n, V = 20000, 12
    x = torch.linspace(-1.0, 1.5, V, device="cuda").repeat(n, 1)
    u = torch.rand(n, generator=torch.Generator(device="cuda").manual_seed(4), device="cuda")
    r = binding.sample_logits(x, u, top_k=8, temperature=0.7)
    p = torch.softmax(x[0, 4:] / 0.7, 0).cpu().double().numpy()
    counts = torch.bincount(r["tokens"].long(), minlength=V).cpu().numpy()
    assert (counts[:4] == 0).all() and (np.abs(counts[4:] - n * p) <= 5 * np.sqrt(n * p * (1 - p))).all()


def test_reports_bad_tokens():
    from paper_2410_17765_b200 import binding

    x, u = draw(3, 100, 0, torch.float32)
    for bad in (-2, 100):
        st = torch.zeros(1, dtype=torch.int32, device="cuda")
        r = binding.sample_logits(x, u, given=torch.tensor([5, bad, -1], dtype=torch.int32, device="cuda"), dev_status=st)
        assert int(st.item()) == 1 and r["logp_given"][1:].tolist() == [-float("inf")] * 2 and np.isfinite(float(r["logp_given"][0]))
