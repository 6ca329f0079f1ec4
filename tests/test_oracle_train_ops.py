"""The fp64 restatement of the training-step operators: gradients against central differences, and the properties of the
8-bit states that the optimiser rests on."""
import numpy as np
import pytest

from oracle import train_ops as T


@pytest.mark.parametrize("gate_kind", ["none", "row", "channel"])
@pytest.mark.parametrize("post", [True, False])
def test_norm_gradients_match_differences(gate_kind, post):
    rng = np.random.default_rng(3)
    N, d = 5, 7
    v = dict(x=rng.normal(size=(N, d)), block=rng.normal(size=(N, d)), w_pre=1 + 0.1 * rng.normal(size=d))
    if post:
        v["w_post"] = 1 + 0.1 * rng.normal(size=d)
    if gate_kind != "none":
        v["gate"] = rng.normal(size=N if gate_kind == "row" else (N, d))
    dy, dx_out = rng.normal(size=(N, d)), rng.normal(size=(N, d))

    def loss(a):
        r = T.norm_forward(a["x"], a["w_pre"], a["block"], a.get("gate"), a.get("w_post"), res_scale=0.7, eps=1e-3)
        return np.sum(r["y"] * dy) + np.sum(r["x_out"] * dx_out)

    f = T.norm_forward(v["x"], v["w_pre"], v["block"], v.get("gate"), v.get("w_post"), res_scale=0.7, eps=1e-3)
    g = T.norm_backward(dy, f["x_out"], v["w_pre"], f["rstd_pre"], dx_out, v["block"], v.get("gate"), v.get("w_post"),
                        f["rstd_post"], res_scale=0.7)
    names = dict(x="dx", block="dblock", w_pre="dw_pre", w_post="dw_post", gate="dgate")
    for key, a in v.items():
        h = 1e-6
        for idx in np.ndindex(a.shape):
            up, dn = ({**v, key: a.copy()} for _ in range(2))
            up[key][idx] += h
            dn[key][idx] -= h
            assert abs((loss(up) - loss(dn)) / (2 * h) - g[names[key]][idx]) < 1e-7, (key, idx)


def test_embed_gradient_is_the_transpose_of_the_lookup():
    rng = np.random.default_rng(0)
    x = np.array([3, -1, 3, 0, 9, -7, 12])         # padding, repeats, clamped on both sides
    E, dy = rng.normal(size=(10, 4)), rng.normal(size=(x.size, 4))
    lhs = np.sum(T.embed_forward(E, x, 1.5) * dy)
    dE, _, _ = T.embed_backward(dy, x, 10, 1.5)
    assert abs(lhs - np.sum(dE * E)) < 1e-12


def test_state_codes_round_trip_and_cover_their_range():
    for second, top in ((False, 128), (True, 256)):
        code = np.zeros(BLOCKS * 256, np.uint8)
        code[:] = np.arange(code.size) % top
        e = np.full(BLOCKS, 120, np.uint8)
        x = T.decode(code, e, second)
        again, e2 = T.encode(x, np.zeros(code.size), second)
        # the largest code leaves no room for a step up: the exponent moves on by one, and the values stay what they were
        assert (e2 == 121).all()
        assert (T.decode(again, e2, second)[16:] <= x[16:]).all()
        assert np.all(np.diff(x[:top]) > 0)
        bits = 4 if second else 3
        assert x[1] / x[top - 1] == 2.0 ** -(14 + bits) / (2 - 2.0 ** -bits)


BLOCKS = 4


def test_state_rounding_keeps_the_mean():
    rng = np.random.default_rng(1)
    x = np.tile(np.exp(rng.normal(size=256) * 2).astype(np.float32), 1)
    for second in (False, True):
        total = np.zeros(256)
        n = 4000
        for s in range(n):
            u = T.noise(256, 5, s).astype(np.int64)
            c, e = T.encode(x, u >> 13 if second else (u & 0xFFFF) << 4, second)
            total += T.decode(c, e, second)
        # one rounding errs by at most one unit, 2^-bits of the value (2^-18 of the block's largest below the normal
        # range), with a standard deviation of at most half of that: five of its standard errors
        unit = np.maximum(x * 2.0 ** -(4 if second else 3), x.max() * 2.0 ** -17)
        assert (np.abs(total / n - x) <= 5 * 0.5 * unit / np.sqrt(n)).all()


def test_eight_bit_states_follow_the_exact_moments():
    """Over 400 steps at beta2 = 0.999, where nearest rounding would stop the second moment at a fraction of its value."""
    rng = np.random.default_rng(2)
    n, betas = 1024, (0.9, 0.999)
    sigma = np.exp(rng.normal(size=n))
    m, v = np.zeros(n, np.uint8), np.zeros(n, np.uint8)
    me, ve = np.zeros(4, np.uint8), np.zeros(4, np.uint8)
    v64 = np.zeros(n)
    for t in range(1, 401):
        g = (sigma * rng.normal(size=n)).astype(np.float32)
        m, me, v, ve = T.adamw_states_8bit(g, m, me, v, ve, betas=betas, step=t, seed=7)
        v64 = betas[1] * v64 + (1 - betas[1]) * g.astype(np.float64) ** 2
    ratio = T.decode(v, ve, True) / v64
    # each step adds a rounding of at most one unit (1/16) with probability p = (change / unit): variance p / 256 a step
    # at a relative change of 2 (1 - beta2) at most on average, over 400 steps: 400 * 0.002 * 16 / 256 = 0.05
    assert abs(ratio.mean() - 1) < 5 * np.sqrt(0.05 / n)
    assert ratio.std() < 2 * np.sqrt(0.05)


def test_blocks_with_infinities_decode_to_nan_and_zero_blocks_to_zero():
    x = np.zeros(512, np.float32)
    x[300] = np.inf
    for second in (False, True):
        c, e = T.encode(x, np.full(512, 7), second)
        y = T.decode(c, e, second)
        assert (y[:256] == 0).all() and np.isnan(y[256:]).all()
