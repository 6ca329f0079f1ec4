"""Paged cache: appending, attention over it and eviction from it, against the fp64 restatement.

Bounds.  A score is a sum of D exact products in fp32, off by (D + 4) 2^-24 of the sum of their magnitudes (`terms`), and so is a weight
p relatively, twice (numerator and denominator), with 2^-21 for the exponential and n 2^-24 for the sum of n of them.  Before the
second product a weight is held as two bf16, 2^-16; the sum over n slots is off by n 2^-24 of sum p |v| (`mass`); out is rounded to
bf16, 2^-8 of its value.  Moved values and selections are exact."""
import numpy as np
import pytest
import torch

from oracle import serve_ops as S

pytestmark = pytest.mark.gpu

NHD, HND = "NHD", "HND"


def numbers(t):
    return t.float().cpu().numpy().astype(np.float64)


class Case:
    """A cache with pages in random places, filled with NaN wherever no sequence has a slot."""

    def __init__(self, lens, H, D, page, *, fresh=None, Q=1, Hq=None, layout=NHD, acc=True, more=0, seed=0, std=1.0):
        rng = np.random.default_rng(seed)
        self.lens, self.H, self.D, self.page, self.Q, self.Hq = lens, H, D, page, Q, Hq or H
        B = len(lens)
        self.fresh = [Q] * B if fresh is None else fresh
        width = max(1, max(-(-n // page) for n in lens)) + 1
        P = B * (width + more) + 2
        place = rng.permutation(P)[:B * (width + more)].reshape(B, width + more).astype(np.int32)
        self.table_np, self.out_np = place[:, :width].copy(), place[:, width:].copy()
        for b, n in enumerate(lens):
            self.table_np[b, -(-n // page):] = -7          # behind the last page the table holds nothing of use
        used = np.zeros((P, page), bool)
        for b, n in enumerate(lens):
            used[S.places(place[b], page, n)] = True
        mask = torch.from_numpy(used).view(P, page, 1, 1)

        def make():
            t = torch.from_numpy(rng.normal(size=(P, page, H, D)).astype(np.float32) * std).masked_fill(~mask, float("nan")).to(torch.bfloat16).cuda()
            return t if layout == NHD else t.transpose(1, 2).contiguous().transpose(1, 2)

        self.k, self.v = make(), make()
        self.acc = None
        if acc:
            self.acc = torch.from_numpy(np.where(used[:, None, :], np.exp(rng.normal(size=(P, H, page))), np.nan).astype(np.float32)).cuda()
        self.table, self.table_out = torch.from_numpy(self.table_np).cuda(), torch.from_numpy(self.out_np).cuda()
        self.lens_t = torch.tensor(lens, dtype=torch.int32, device="cuda")
        self.fresh_t = None if fresh is None else torch.tensor(fresh, dtype=torch.int32, device="cuda")
        self.q = torch.from_numpy(rng.normal(size=(B, Q, self.Hq, D)).astype(np.float32)).to(torch.bfloat16).cuda()
        self.status = torch.zeros(1, dtype=torch.int32, device="cuda")

    def cache(self):
        from paper_2410_17765_b200 import binding

        return binding.PagedCache(self.k, self.v, self.acc)

    def of(self, cache, b):
        """[n, H, D] of sequence b."""
        page, at = S.places(self.table_np[b], self.page, self.lens[b])
        return numbers(cache)[page, at]


def check_attend(c, *, scale=None, want_acc=True, q=None):
    from paper_2410_17765_b200 import binding

    q = c.q if q is None else q
    B, Q, Hq, D = q.shape
    before = None if c.acc is None else c.acc.clone()
    out = dict(out=torch.full((B, Q, Hq, D), 77.0, dtype=torch.bfloat16, device="cuda"), lse=torch.full((B, Q, Hq), 77.0, device="cuda"))
    binding.cache_attend(c.cache(), q, c.table, c.lens_t, q_lens=c.fresh_t, scale=scale, out=out, accumulate=want_acc, dev_status=c.status)
    assert int(c.status.item()) == 0
    scale = D ** -0.5 if scale is None else scale
    got, lse = numbers(out["out"]), out["lse"].cpu().numpy().astype(np.float64)
    want_acc_np = None if before is None else before.cpu().numpy().astype(np.float64)
    acc_tol = None if before is None else np.zeros_like(want_acc_np)
    for b in range(B):
        n, fresh = c.lens[b], c.fresh[b]
        K, V = c.of(c.k, b), c.of(c.v, b)
        r = S.attend(numbers(q[b]), K, V, fresh, scale)
        p_rel = 2 * (D + 4) * 2.0 ** -24 * r["terms"] + 2.0 ** -20 + n * 2.0 ** -24
        tol = 2.0 ** -8 * np.abs(r["out"]) + r["mass"] * (p_rel + 2.0 ** -16 + n * 2.0 ** -24)[:, :, None] + 1e-37
        assert (np.abs(got[b, :fresh] - r["out"]) <= tol).all(), (b, np.abs(got[b, :fresh] - r["out"]).max())
        empty = np.isneginf(r["lse"])
        assert np.isneginf(lse[b, :fresh][empty]).all()
        seen = ~empty
        assert (np.abs(lse[b, :fresh][seen] - r["lse"][seen]) <= p_rel[seen] + 2.0 ** -22 * np.abs(r["lse"][seen])).all()
        assert (got[b, fresh:] == 77).all() and (lse[b, fresh:] == 77).all()
        if before is not None and want_acc:
            page, at = S.places(c.table_np[b], c.page, n)
            want_acc_np[page, :, at] += r["weights"].T
            acc_tol[page, :, at] = (r["weights"] * (p_rel.max() if p_rel.size else 0)).T + 2.0 ** -23 * np.abs(want_acc_np[page, :, at])
    if before is not None:
        acc = c.acc.cpu().numpy().astype(np.float64)
        assert np.array_equal(np.isnan(acc), np.isnan(want_acc_np))
        fine = ~np.isnan(acc)
        assert (np.abs(acc - want_acc_np)[fine] <= acc_tol[fine]).all()
    return out


EDGES = [0, 1, 2, 7, 8, 9, 63, 64, 65, 127, 128, 129, 255, 256, 257, 1000]


@pytest.mark.parametrize("layout", [NHD, HND])
@pytest.mark.parametrize("page", [8, 16, 24, 64, 128, 256, 1000])
def test_attend_lengths_and_pages(page, layout):
    check_attend(Case(EDGES, 2, 64, page, Hq=4, layout=layout, seed=page))


@pytest.mark.parametrize("D", [8, 16, 24, 40, 64, 72, 80, 96, 120, 128])
def test_attend_widths(D):
    check_attend(Case([300, 1, 130], 3, D, 32, Hq=6, seed=D))


@pytest.mark.parametrize("H,Hq", [(1, 1), (1, 7), (8, 8), (2, 32), (1, 64), (3, 39), (1, 200)])
def test_attend_heads(H, Hq):
    check_attend(Case([513, 40, 129], H, 64, 16, Hq=Hq, seed=Hq))


@pytest.mark.parametrize("Q,fresh", [(1, [0, 1, 1]), (5, [5, 0, 3]), (9, [9, 9, 1]), (33, [33, 2, 17]), (130, [130, 129, 1])])
@pytest.mark.parametrize("layout", [NHD, HND])
def test_attend_drafts(Q, fresh, layout):
    check_attend(Case([700, 131, 20], 2, 128, 64, Hq=8, Q=Q, fresh=fresh, layout=layout, seed=Q))


def test_attend_tokens_that_see_nothing():
    check_attend(Case([0, 2, 5], 2, 64, 8, Hq=4, Q=5, seed=3))


@pytest.mark.parametrize("B,n", [(1, 20000), (3, 9000), (70, 700), (300, 33)])
def test_attend_shares_of_the_work(B, n):
    rng = np.random.default_rng(B)
    check_attend(Case([n] + [int(v) for v in rng.integers(1, n, B - 1)], 2, 64, 64, Hq=4, seed=B))


def test_attend_without_weights():
    check_attend(Case([100, 300], 2, 64, 16, Hq=4, acc=False))
    check_attend(Case([100, 300], 2, 64, 16, Hq=4), want_acc=False)


@pytest.mark.parametrize("H,Hq,D,lens,Q", [(2, 4, 128, [300, 131, 3], 5), (1, 1, 64, [258, 129, 40], 3), (2, 6, 72, [5000, 130, 0], 7), (1, 8, 40, [700, 300, 64], 45)])
@pytest.mark.parametrize("of", ["keys", "values"])
def test_attend_infinities_and_nan_reach_the_tokens_that_see_them(H, Hq, D, lens, Q, of):
    """Slots of the new tokens hold them; some of the tokens see none of these slots, some one, some more.

    Values leave the scores alone, so that the other tokens' bits stay.  Keys that are infinite may move the references that weights are taken
    relative to: a weight is then off by 2^-20 + 2^-16, a sum of 5000 by 2 * 5000 * 2^-24 of mass <= 5, which is below 2^-7, and each result by 2^-8."""
    from paper_2410_17765_b200 import binding

    c = Case(lens, H, D, 16, Hq=Hq, Q=Q, seed=Q)
    rng = np.random.default_rng(D)
    where = []
    for b, n in enumerate(lens):
        for value in (float("inf"), float("-inf"), float("nan")):
            slot, h, col = n - 1 - int(rng.integers(0, Q - 1)), int(rng.integers(0, H)), int(rng.integers(0, D))
            if slot < 0:
                continue
            page, at = S.places(c.table_np[b], c.page, n)
            where.append((h, col, value, int(page[slot]), int(at[slot])))
    plain = check_attend(c, want_acc=False)
    target = c.k if of == "keys" else c.v
    for h, col, value, page, at in where:
        target[page, at, h, col] = value
    c.acc.zero_()
    got = binding.cache_attend(c.cache(), c.q, c.table, c.lens_t, accumulate=True, dev_status=c.status)
    assert int(c.status.item()) == 0
    got, plain, acc, G = numbers(got["out"]), numbers(plain["out"]), numbers(c.acc), Hq // H
    for b, n in enumerate(lens):
        K, V = c.of(c.k, b), c.of(c.v, b)
        for j in range(Q):
            seen = max(0, n - (Q - 1 - j))
            for hq in range(Hq):
                h = hq // G
                row, was = got[b, j, hq], plain[b, j, hq]
                if np.isfinite(K[:seen, h]).all() and np.isfinite(V[:seen, h]).all():
                    assert np.array_equal(row, was) if of == "values" else (np.abs(row - was) <= 2.0 ** -7 * np.abs(was) + 2.0 ** -7).all()
                elif of == "values":
                    want = np.where(np.isfinite(V[:seen, h]), 0.0, V[:seen, h]).sum(0)        # inf - inf is NaN
                    assert np.array_equal(np.isnan(row), np.isnan(want))
                    assert np.array_equal(row[np.isinf(want)], want[np.isinf(want)])
                    assert np.array_equal(row[want == 0], was[want == 0])
        if of == "values" and n:
            page, at = S.places(c.table_np[b], c.page, n)
            assert np.allclose(acc[page, :, at].sum(0), G * min(n, Q), rtol=2.0 ** -10)


@pytest.mark.parametrize("std", [1e-3, 8.0, 60.0])
def test_attend_scales(std):
    """Flat maps, and maps of one slot; a scale of its own, also a negative one."""
    check_attend(Case([900, 129], 2, 64, 64, Hq=4, std=std))
    check_attend(Case([900, 129], 2, 64, 64, Hq=4, std=std), scale=-0.3)


def test_attend_rising_scores():
    """The running maximum changes in every tile, and once by far."""
    c = Case([1500], 1, 64, 64, Hq=2, seed=5)
    page, at = S.places(c.table_np[0], 64, 1500)
    ramp = torch.linspace(-40, 40, 1500).to(torch.bfloat16).cuda()
    c.k[page, at, 0] = 0
    c.k[page, at, 0, 0] = ramp
    c.k[page[1400], at[1400], 0, 0] = 3000.0
    c.q.zero_()
    c.q[..., 0] = 1.0
    check_attend(c, scale=1.0)


@pytest.mark.parametrize("shift", [0, 1, 3])
def test_attend_strided_queries_and_outputs(shift):
    """Slices of a projection whose rows start at any element."""
    from paper_2410_17765_b200 import binding

    c = Case([200, 90], 2, 64, 16, Hq=4, Q=3, fresh=[3, 2])
    wide = torch.randn(2, 3, 1000, device="cuda").to(torch.bfloat16)
    q = wide[:, :, shift:shift + 256].view(2, 3, 4, 64) if shift == 0 else wide[:, :, shift:shift + 256].unflatten(2, (4, 64))
    q.copy_(c.q)
    check_attend(c, q=q)
    room = torch.full((2, 3, 1000), 5.0, dtype=torch.bfloat16, device="cuda")
    out = room[:, :, shift:shift + 256].unflatten(2, (4, 64))
    want = binding.cache_attend(c.cache(), c.q, c.table, c.lens_t, q_lens=c.fresh_t)["out"]
    binding.cache_attend(c.cache(), q, c.table, c.lens_t, q_lens=c.fresh_t, out=dict(out=out))
    assert torch.equal(out[0], want[0]) and torch.equal(out[1, :2], want[1, :2])
    assert (out[1, 2] == 5).all() and (room[:, :, :shift] == 5).all() and (room[:, :, shift + 256:] == 5).all()


def test_attend_of_a_cache_in_one_tensor():
    """Keys and values interleaved in one allocation, with room between the heads."""
    from paper_2410_17765_b200 import binding

    c = Case([333, 65], 2, 40, 24, Hq=4)
    both = torch.full((c.k.shape[0], 2, 24, 2, 48), float("nan"), dtype=torch.bfloat16, device="cuda")
    both[:, 0, :, :, :40], both[:, 1, :, :, :40] = c.k, c.v
    want = binding.cache_attend(c.cache(), c.q, c.table, c.lens_t, accumulate=False)["out"]
    got = binding.cache_attend(binding.PagedCache(both[:, 0, :, :, :40], both[:, 1, :, :, :40]), c.q, c.table, c.lens_t)["out"]
    assert torch.equal(got, want)


def test_attend_bits_repeat():
    from paper_2410_17765_b200 import binding

    c = Case([777, 1300, 64], 2, 64, 64, Hq=8, acc=False)
    a = binding.cache_attend(c.cache(), c.q, c.table, c.lens_t, want_lse=True)
    b = binding.cache_attend(c.cache(), c.q, c.table, c.lens_t, want_lse=True)
    assert torch.equal(a["out"], b["out"]) and torch.equal(a["lse"], b["lse"])


def test_attend_reports_bad_tables_and_lengths():
    from paper_2410_17765_b200 import binding

    c = Case([300, 20], 2, 64, 16, Hq=4, acc=True)
    for bad in (-1, 10 ** 6):
        t = c.table.clone()
        t[0, 3] = bad
        c.status.zero_()
        r = binding.cache_attend(c.cache(), c.q, t, c.lens_t, dev_status=c.status)
        assert int(c.status.item()) == 1 and torch.isfinite(r["out"]).all()
    for bad in (-5, 10 ** 8):
        n = c.lens_t.clone()
        n[1] = bad
        t = c.table.clamp(min=0)
        c.status.zero_()
        binding.cache_attend(c.cache(), c.q, t, n, dev_status=c.status, accumulate=False)
        assert int(c.status.item()) == 1
    c.status.zero_()
    binding.cache_attend(c.cache(), c.q, c.table, c.lens_t, q_lens=torch.tensor([1, 4], dtype=torch.int32, device="cuda"), dev_status=c.status)
    assert int(c.status.item()) == 1


@pytest.mark.parametrize("layout", [NHD, HND])
@pytest.mark.parametrize("H,D,page,shift", [(1, 8, 8, 0), (2, 64, 16, 0), (5, 80, 24, 1), (8, 128, 256, 4)])
def test_append(H, D, page, layout, shift):
    from paper_2410_17765_b200 import binding

    lens, fresh = [40, 7, 300, 9, 100], [40, 7, 21, 0, 1]
    c = Case(lens, H, D, page, Q=40, fresh=fresh, layout=layout)
    both = torch.randn(5, 40, 2 * H * D + 16, device="cuda").to(torch.bfloat16)
    k, v = both[:, :, shift:shift + H * D].unflatten(2, (H, D)), both[:, :, H * D + shift:2 * H * D + shift].unflatten(2, (H, D))
    want_k, want_v, want_a = c.k.clone(), c.v.clone(), c.acc.clone()
    for b, (n, f) in enumerate(zip(lens, fresh)):
        pg, at = (torch.from_numpy(x.astype(np.int64)).cuda() for x in S.places(c.table_np[b], page, n))
        want_k[pg[n - f:], at[n - f:]], want_v[pg[n - f:], at[n - f:]] = k[b, :f], v[b, :f]
        want_a[pg[n - f:], :, at[n - f:]] = 0
    binding.cache_append(c.cache(), k, v, c.table, c.lens_t, q_lens=c.fresh_t, dev_status=c.status)
    assert int(c.status.item()) == 0
    for got, want in ((c.k, want_k), (c.v, want_v), (c.acc, want_a)):
        assert torch.equal(torch.nan_to_num(got, 99.0), torch.nan_to_num(want, 99.0))


def test_append_leaves_out_what_has_no_slot():
    from paper_2410_17765_b200 import binding

    c = Case([40, 20], 2, 64, 16, Q=4)
    k = torch.randn(2, 4, 2, 64, device="cuda").to(torch.bfloat16)
    before = c.k.clone()
    for lens, table in (([2, 10 ** 6], c.table), ([40, 20], torch.full_like(c.table, -1)), ([-3, -3], c.table)):
        c.status.zero_()
        n = torch.tensor(lens, dtype=torch.int32, device="cuda")
        t = table.clone()
        t[1] = -1
        binding.cache_append(c.cache(), k, k, t, n, dev_status=c.status)
        assert int(c.status.item()) == 1
    pg, at = S.places(c.table_np[0], 16, 2)
    before[torch.from_numpy(pg.astype(np.int64)).cuda(), torch.from_numpy(at).cuda()] = k[0, 2:]
    assert torch.equal(torch.nan_to_num(c.k, 99.0), torch.nan_to_num(before, 99.0))


def check_evict(c, budget, recent):
    from paper_2410_17765_b200 import binding

    k0, v0, a0 = c.k.clone(), c.v.clone(), c.acc.clone()
    acc = c.acc.cpu().numpy()
    r = binding.cache_evict(c.cache(), c.table, c.lens_t, c.table_out, budget, recent=recent, dev_status=c.status)
    assert int(c.status.item()) == 0
    assert r["lens"].tolist() == [min(n, budget) for n in c.lens]
    kept = r["kept"].cpu().numpy()
    for b, n in enumerate(c.lens):
        m = min(n, budget)
        page, at = S.places(c.table_np[b], c.page, n)
        to, into = S.places(c.out_np[b], c.page, m)
        for h in range(c.H):
            want = S.evict(acc[page, h, at], n, budget, recent)
            assert kept[b, h, :m].tolist() == want.tolist() and (kept[b, h, m:] == -1).all()
            for new, old in ((k0, c.k), (v0, c.v)):
                new[torch.from_numpy(to.astype(np.int64)), torch.from_numpy(into), h] = old[torch.from_numpy(page[want].astype(np.int64)), torch.from_numpy(at[want]), h]
            a0[torch.from_numpy(to.astype(np.int64)), h, torch.from_numpy(into)] = c.acc[torch.from_numpy(page[want].astype(np.int64)), h, torch.from_numpy(at[want])]
    for got, want in ((c.k, k0), (c.v, v0), (c.acc, a0)):
        assert torch.equal(torch.nan_to_num(got, 99.0), torch.nan_to_num(want, 99.0))


@pytest.mark.parametrize("layout", [NHD, HND])
@pytest.mark.parametrize("H,D,page,budget,recent", [(1, 8, 8, 1, 0), (1, 8, 8, 1, 1), (3, 64, 16, 100, 0), (2, 80, 24, 100, 30), (2, 128, 64, 257, 257),
                                                    (8, 64, 256, 1000, 100)])
def test_evict(H, D, page, budget, recent, layout):
    check_evict(Case([0, 1, budget - 1, budget, budget + 1, 3 * budget + 5, 2000], H, D, page, layout=layout, more=-(-budget // page), seed=budget), budget, recent)


@pytest.mark.parametrize("kind", ["equal", "zeros", "few", "nan", "infinite", "signed"])
def test_evict_ties_and_odd_weights(kind):
    c = Case([1500, 700, 3000], 2, 16, 32, more=20, seed=4)
    g = torch.Generator(device="cuda").manual_seed(1)
    r = torch.rand(c.acc.shape, generator=g, device="cuda")
    c.acc.copy_({"equal": torch.full_like(r, 0.5), "zeros": torch.where(r < 0.7, 0.0, r), "few": (r * 3).floor(), "nan": torch.where(r < 0.6, float("nan"), r),
                 "infinite": torch.where(r < 0.3, float("inf"), torch.where(r > 0.6, -float("inf"), r)), "signed": torch.where(r < 0.5, -0.0, (r - 0.7) * 1e-40)}[kind])
    check_evict(c, 600, 50)


def test_evict_long_sequences():
    check_evict(Case([70000, 50001, 3], 1, 16, 64, more=40, seed=9), 2000, 77)


def test_evict_reports_bad_tables():
    from paper_2410_17765_b200 import binding

    c = Case([300, 200], 2, 16, 16, more=4)
    for which in (c.table, c.table_out):
        keep = int(which[1, 1])
        for bad in (-1, 10 ** 6):
            which[1, 1] = bad
            c.status.zero_()
            r = binding.cache_evict(c.cache(), c.table, c.lens_t, c.table_out, 64, recent=8, dev_status=c.status)
            assert int(c.status.item()) == 1 and r["lens"].tolist() == [64, 64]
        which[1, 1] = keep
