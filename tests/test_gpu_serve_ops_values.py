"""Values at the ends of their range in the serving operators: what infinities, NaN and the largest scores come out as."""
import numpy as np
import pytest
import torch

from oracle import serve_ops as S
from test_gpu_cache import Case, check_attend, numbers

pytestmark = pytest.mark.gpu

INF, NAN = float("inf"), float("nan")


@pytest.mark.parametrize("std", [1.0, 60.0])           # (60: nearly all weights underflow)
@pytest.mark.parametrize("H,Hq,D,page,lens,Q", [(2, 4, 128, 16, [300, 131, 1], 1), (1, 1, 64, 8, [258, 129, 40], 1), (2, 6, 72, 24, [5000, 130, 0], 7), (1, 8, 40, 64, [700, 300, 64], 45),
                                                (1, 2, 128, 64, [40000], 3), (1, 20, 128, 256, [30000, 513], 1)])
def test_infinite_values_of_older_slots_come_out_as_they_are(H, Hq, D, page, lens, Q, std):
    """Every token sees these slots: the columns that hold them are infinite or NaN for all tokens, as their sum is, whatever the weights; all other bits stay."""
    from paper_2410_17765_b200 import binding

    c = Case(lens, H, D, page, Hq=Hq, Q=Q, seed=Q + D, std=std, acc=False)
    plain = check_attend(c)
    rng = np.random.default_rng(D)
    for b, n in enumerate(lens):
        old = n - Q + 1                                  # slots that all tokens see
        if old <= 0:
            continue
        page_of, at = S.places(c.table_np[b], page, n)
        slots = [0, old - 1] + [int(s) for s in rng.integers(0, old, 6)]
        for col, kinds in enumerate([(INF,), (-INF,), (NAN,), (INF, -INF), (INF, INF), (-INF, -INF), (INF, NAN)]):
            for value in kinds:
                slot = slots[int(rng.integers(0, len(slots)))]
                c.v[int(page_of[slot]), int(at[slot]), int(rng.integers(0, H)), col] = value
        if Q > 1:                                        # one of both kinds, and in the slots of the draft as well
            c.v[int(page_of[0]), int(at[0]), 0, D - 1] = INF
            c.v[int(page_of[n - 1]), int(at[n - 1]), 0, D - 1] = -INF
    out = {"lse": torch.zeros(len(lens), Q, Hq, device="cuda")}
    got = numbers(binding.cache_attend(c.cache(), c.q, c.table, c.lens_t, out=out, dev_status=c.status)["out"])
    assert int(c.status.item()) == 0 and torch.equal(out["lse"], plain["lse"])
    was = numbers(plain["out"])
    met = set()
    for b, n in enumerate(lens):
        V = c.of(c.v, b)
        for j in range(Q):
            seen = max(0, n - (Q - 1 - j))
            for hq in range(Hq):
                v = V[:seen, hq // (Hq // H)]
                with np.errstate(invalid="ignore"):
                    want = np.where(np.isfinite(v), 0.0, v).sum(0)
                row = got[b, j, hq]
                met |= set(want[want != 0].tolist())
                assert np.array_equal(np.isnan(row), np.isnan(want)), (b, j, hq)
                assert np.array_equal(row[np.isinf(want)], want[np.isinf(want)])
                assert np.array_equal(row[want == 0], was[b, j, hq][want == 0])
    assert INF in met and -INF in met


def test_values_that_overflow_or_are_nan_by_their_weights_stay_so():
    """A key of NaN: its row's results are NaN in every column, with and without an infinite value beside it."""
    from paper_2410_17765_b200 import binding

    c = Case([200, 90], 1, 64, 16, Hq=4, seed=1, acc=False)
    page, at = S.places(c.table_np[0], 16, 200)
    c.k[int(page[5]), int(at[5]), 0, 3] = NAN
    c.v[int(page[9]), int(at[9]), 0, 7] = INF
    got = numbers(binding.cache_attend(c.cache(), c.q, c.table, c.lens_t)["out"])
    assert np.isnan(got[0]).all() and np.isfinite(got[1]).all()


@pytest.mark.parametrize("H,Hq,D,page,lens,Q", [(2, 4, 64, 16, [300, 131, 6], 5), (1, 8, 128, 64, [20000, 64], 9), (1, 2, 40, 8, [129], 3)])
@pytest.mark.parametrize("bad", [NAN, INF])
def test_a_broken_query_adds_to_the_slots_that_it_sees_alone(bad, H, Hq, D, page, lens, Q):
    """The query of one token is NaN or infinite: its weights are NaN.  Slots behind it get the later tokens' weights, within the bounds of the others."""
    from paper_2410_17765_b200 import binding

    c = Case(lens, H, D, page, Hq=Hq, Q=Q, seed=D)
    broken = Q // 2 - 1
    c.q[:, broken, :, 1] = bad
    before = numbers(c.acc)
    binding.cache_attend(c.cache(), c.q, c.table, c.lens_t, dev_status=c.status)
    assert int(c.status.item()) == 0
    after = numbers(c.acc)
    for b, n in enumerate(lens):
        page_of, at = S.places(c.table_np[b], page, n)
        sees = max(0, n - (Q - 1 - broken))
        got, was = after[page_of, :, at], before[page_of, :, at]
        assert np.isnan(got[:sees]).all()
        # the tokens behind the broken one alone: its own rows and those before it have no weight there
        later = S.attend(numbers(c.q[b, broken + 1:]), c.of(c.k, b), c.of(c.v, b), Q - 1 - broken, D ** -0.5)
        p_rel = 2 * (D + 4) * 2.0 ** -24 * later["terms"].max() + 2.0 ** -20 + n * 2.0 ** -24
        want = was[sees:] + later["weights"].T[sees:]
        assert len(want) and (np.abs(got[sees:] - want) <= later["weights"].T[sees:] * p_rel + 2.0 ** -23 * np.abs(want)).all()


@pytest.mark.parametrize("n,Q", [(1, 1), (40, 3), (300, 1), (20000, 2)])
@pytest.mark.parametrize("top", [126, -126])
def test_scores_near_the_ends_of_fp32(top, n, Q):
    """Scores of about +-2^126.9 (in units of log 2 +-2^127.4, still finite), one of them nearer to zero by a factor that leaves the others no weight: its value comes
    out, rounded by 2^-24 for the product of a weight of one and its sum, and 2^-8."""
    from paper_2410_17765_b200 import binding

    c = Case([n], 1, 8, 16, Hq=2, Q=Q, seed=n)
    page, at = S.places(c.table_np[0], 16, n)
    page, at = torch.from_numpy(page.astype(np.int64)).cuda(), torch.from_numpy(at).cuda()
    c.q.zero_()
    c.q[..., 0] = 2.0 ** 63
    c.k[page, at] = 0.0
    big = 1.875 * 2.0 ** (abs(top) - 63)
    best = 0 if top < 0 or n == 1 else n // 2
    c.k[page, at, 0, 0] = -big
    c.k[page[best], at[best], 0, 0] = (big if top > 0 else -big) * 0.9375
    before = c.acc.clone()
    r = binding.cache_attend(c.cache(), c.q, c.table, c.lens_t, scale=1.0, want_lse=True, dev_status=c.status)
    assert int(c.status.item()) == 0
    got, value = numbers(r["out"])[0], numbers(c.v)[int(page[best]), int(at[best]), 0]
    score = 2.0 ** 63 * float(c.k[page[best], at[best], 0, 0])
    for j in range(Q):
        if best < n - (Q - 1 - j):
            assert (np.abs(got[j] - value) <= (2.0 ** -8 + 2.0 ** -20) * np.abs(value)).all()
            assert (np.abs(r["lse"][0, j].cpu().numpy().astype(np.float64) - score) <= 2.0 ** -21 * abs(score)).all()
    acc = numbers(c.acc - before)[page.cpu().numpy(), 0, at.cpu().numpy()]
    seen = sum(best < n - (Q - 1 - j) for j in range(Q))
    assert abs(acc[best] - 2 * seen) <= 2.0 ** -18 and (np.delete(acc, best) == 0).all()


@pytest.mark.parametrize("how,left", [(dict(), None), (dict(top_p=0.9), 3), (dict(top_k=3), 3), (dict(min_p=0.5), 3), (dict(top_k=4, top_p=0.6), 2), (dict(top_k=2), 2)], ids=str)
@pytest.mark.parametrize("V", [5, 3001])
def test_the_largest_number_beside_an_infinite_logit_counts_as_infinite(V, how, left):
    """Three entries share the mass: `left` of them, and nothing else, are left by a filter (without one every entry is).  Drawn and given tokens have the log-probability of the share that they were drawn with."""
    from paper_2410_17765_b200 import binding

    big = torch.finfo(torch.float32).max
    x = torch.zeros(8, V, device="cuda")
    x[:, 1], x[:, 2], x[:, 4] = big, INF, big
    u = (torch.arange(8, device="cuda") + 0.5) / 8
    given = torch.tensor([1, 2, 4, 0, 1, 2, 4, 3], dtype=torch.int32, device="cuda")
    r = binding.sample_logits(x, u, given=given, want_kept=True, **how)
    assert r["kept"].tolist() == [V if left is None else left] * 8
    kept = 3 if left is None else left
    order = [2, 1, 4][:kept]                               # by falling logits, of equals the first
    assert set(r["tokens"].tolist()) == set(order)
    want = torch.full((8,), -float(np.log(kept)), device="cuda")
    assert (r["logp"] - want).abs().max() <= 2.0 ** -22
    for g, got in zip(given.tolist(), r["logp_given"].tolist()):
        assert abs(got + np.log(kept)) <= 2.0 ** -22 if g in order else got == -INF


@pytest.mark.parametrize("how", [dict(p=0.95), dict(p=0.3), dict(p=0.999, T=1e-3), dict(p=0.9, min_p=0.5), dict(p=0.9, k=700), dict(T=1e20, p=0.6)], ids=str)
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("V", [1, 2, 3, 8, 1001, 60000])
def test_rows_that_hold_the_lowest_number_alone(V, dtype, how):
    """Rows that a mask of the type's lowest value leaves nothing of: their entries share the mass, and nothing beside the row counts."""
    from test_gpu_sample import check

    low = torch.finfo(dtype).min
    wide = torch.full((6, V + 5), 3.0, device="cuda", dtype=dtype)
    x = wide[:, 1:1 + V]
    x[:] = low
    x[3, V // 2:] = -INF
    x[4, ::2] = NAN
    x[5, V - 1] = 0.5
    u = torch.tensor([0.0, 0.4, 0.99, 0.7, 0.2, 0.6], device="cuda")
    check(x, u, sure=False, given=torch.full((6,), V - 1, dtype=torch.int32, device="cuda"), **how)


@pytest.mark.parametrize("V", [6, 4001])
def test_infinite_temperatures_of_rows(V):
    """Every kept entry has the same share; beside infinite logits no finite one has any."""
    from paper_2410_17765_b200 import binding

    x = torch.randn(4, V, generator=torch.Generator(device="cuda").manual_seed(V), device="cuda")
    x[2:, 1] = x[2:, 3] = INF
    x[1, 0] = -INF
    given = torch.tensor([V - 1, V - 1, 2, 3], dtype=torch.int32, device="cuda")
    r = binding.sample_logits(x, torch.full((4,), 0.6, device="cuda"), temperature=torch.full((4,), INF, device="cuda"), given=given, want_kept=True)
    assert r["tokens"][2:].tolist() == [3, 3] and r["kept"].tolist() == [V, V - 1, V, V]
    for got, share in ((r["logp"], [V, V - 1, 2, 2]), (r["logp_given"], [V, V - 1, INF, 2])):
        for value, n in zip(got.tolist(), share):
            assert value == -INF if n == INF else abs(value + np.log(n)) <= 2.0 ** -24 * np.log(n) + 2.0 ** -30
