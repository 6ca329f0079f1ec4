"""The fp64 restatement of the serving operators against hand-worked examples and against itself in another form."""
import numpy as np
import pytest

from oracle import serve_ops as S


def test_attend_is_a_weighted_mean_of_what_a_token_sees():
    rng = np.random.default_rng(0)
    q, K, V = rng.normal(size=(3, 4, 8)), rng.normal(size=(6, 2, 8)), rng.normal(size=(6, 2, 8))
    r = S.attend(q, K, V, 3, 0.25)
    for j in range(3):
        for h in range(4):
            s = np.array([0.25 * sum(q[j, h, d] * K[i, h // 2, d] for d in range(8)) for i in range(4 + j)])
            p = np.exp(s) / np.exp(s).sum()
            assert np.allclose(r["out"][j, h], sum(p[i] * V[i, h // 2] for i in range(4 + j)))
            assert np.isclose(r["lse"][j, h], np.log(np.exp(s).sum()))
    assert np.allclose(r["weights"].sum(), 3 * 4)
    assert (r["weights"][:, 5] > 0).all()


def test_attend_of_tokens_that_see_nothing():
    r = S.attend(np.ones((3, 1, 8)), np.ones((1, 1, 8)), np.ones((1, 1, 8)), 3, 1.0)
    assert (r["out"][:2] == 0).all() and np.isneginf(r["lse"][:2]).all() and (r["out"][2] == 1).all()


def test_evict_keeps_recent_and_heavy_slots_and_breaks_ties_to_the_front():
    acc = np.array([1.0, 5.0, 1.0, np.nan, 1.0, 0.0, 9.0, 0.0])
    assert S.evict(acc, 8, 8, 0).tolist() == list(range(8))
    assert S.evict(acc, 8, 4, 1).tolist() == [0, 1, 6, 7]
    assert S.evict(acc, 8, 5, 1).tolist() == [0, 1, 2, 6, 7]
    assert S.evict(acc, 8, 3, 3).tolist() == [5, 6, 7]
    assert S.evict(acc, 8, 7, 0).tolist() == [0, 1, 2, 4, 5, 6, 7]


@pytest.mark.parametrize("u,token", [(0.0, 0), (0.49, 0), (0.51, 2), (0.99, 2)])
def test_sample_draws_by_index_among_the_kept(u, token):
    x = np.log(np.array([4.0, 1.0, 4.0, 2.0]))
    r = S.sample(x, u, 1.0, 2, 1.0, 0.0)
    assert r["token"] == token and r["kept"] == 2 and np.isclose(r["logp"], np.log(0.5))


def test_sample_filters():
    x = np.log(np.array([8.0, 4.0, 2.0, 1.0, 1.0]))
    assert S.sample(x, 0.0, 1.0, 0, 0.5, 0.0)["kept"] == 1
    assert S.sample(x, 0.0, 1.0, 0, 0.51, 0.0)["kept"] == 2
    assert S.sample(x, 0.0, 1.0, 0, 0.93, 0.0)["kept"] == 4          # of the two equals the first
    assert S.sample(x, 0.0, 1.0, 0, 1.0, 0.25)["kept"] == 3
    assert S.sample(x, 0.0, 1.0, 2, 0.9, 0.0)["kept"] == 2           # 0.9 of the mass of two
    assert S.sample(x, 0.9, 0.0, 0, 1.0, 0.0)["token"] == 0
    assert S.sample(np.array([-np.inf, np.nan]), 0.5, 1.0, 0, 1.0, 0.0)["token"] == -1
    r = S.sample(np.array([0.0, np.inf, 1.0, np.inf]), 0.6, 1.0, 0, 1.0, 0.0)
    assert r["token"] == 3 and np.isclose(r["logp"], -np.log(2))
