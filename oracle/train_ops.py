"""fp64 restatement of the operators around the head in a training step: embedding lookup and its gradient, norms with
gate and residual addition, AdamW with fp32 or 8-bit states.  NumPy only.

The 8-bit states' rounding is defined on fp32 values with an integer hash as the noise, so that part works on fp32
arrays step by step and is meant to be matched bit for bit."""
from __future__ import annotations

import numpy as np

BLOCK = 256
U32 = np.uint64(0xFFFFFFFF)


# ---------------------------------------------------------------------------------------------------- embedding
def embed_forward(E, x, scale):
    E, x = np.asarray(E, np.float64), np.asarray(x)
    out = np.zeros((x.size, E.shape[1]))
    for i, v in enumerate(x.ravel()):
        if v != -1:
            out[i] = scale * E[min(max(int(v), 0), E.shape[0] - 1)]
    return out


def embed_backward(dy, x, V, scale, base=None):
    """(dE, sum of magnitudes, number of terms per row)."""
    dy, x = np.asarray(dy, np.float64), np.asarray(x).ravel()
    dE = np.zeros((V, dy.shape[1])) if base is None else np.array(base, np.float64)
    mag, terms = np.abs(dE), np.zeros(V)
    for i, v in enumerate(x):
        if v != -1:
            v = min(max(int(v), 0), V - 1)
            dE[v] += scale * dy[i]
            mag[v] += abs(scale) * np.abs(dy[i])
            terms[v] += 1
    return dE, mag, terms


# ---------------------------------------------------------------------------------------------------- norms
def sigmoid(z):
    with np.errstate(over="ignore"):
        return 1.0 / (1.0 + np.exp(-np.asarray(z, np.float64)))


def _gate(gate, sign=1):
    """The gate; sign -1: one minus it, which the difference would lose above a logit of 37."""
    if gate is None:
        return np.ones((1, 1))
    g = sigmoid(sign * np.asarray(gate, np.float64))
    return g[:, None] if g.ndim == 1 else g


def norm_forward(x, w_pre=None, block=None, gate=None, w_post=None, res_scale=1.0, eps=1e-6):
    x = np.asarray(x, np.float64)
    rb = rx = y = None
    if block is not None:
        u = np.asarray(block, np.float64)
        if w_post is not None:
            rb = (np.mean(u * u, 1) + eps) ** -0.5
            u = u * rb[:, None] * np.asarray(w_post, np.float64)
        x = res_scale * x + _gate(gate) * u
    if w_pre is not None:
        rx = (np.mean(x * x, 1) + eps) ** -0.5
        y = x * rx[:, None] * np.asarray(w_pre, np.float64)
    return dict(x_out=x, y=y, rstd_post=rb, rstd_pre=rx)


def norm_backward(dy, x_out, w_pre=None, rstd_pre=None, dx_out=None, block=None, gate=None, w_post=None, rstd_post=None,
                  res_scale=1.0):
    """Gradients, and under "mag" for each the sum of the magnitudes of its terms: what rounding errors scale with."""
    x = np.asarray(x_out, np.float64)
    N, d = x.shape
    t = np.zeros((N, d)) if dx_out is None else np.asarray(dx_out, np.float64).copy()
    tm = np.abs(t)
    r, mag = {}, {}
    if dy is not None:
        dy, w, rx = np.asarray(dy, np.float64), np.asarray(w_pre, np.float64), np.asarray(rstd_pre, np.float64)[:, None]
        xh = x * rx
        t += rx * (w * dy - xh * np.mean(w * dy * xh, 1, keepdims=True))
        tm += rx * (np.abs(w * dy) + np.abs(xh) * np.mean(np.abs(w * dy * xh), 1, keepdims=True))
        r["dw_pre"], mag["dw_pre"] = np.sum(dy * xh, 0), np.sum(np.abs(dy * xh), 0)
    r["dx"], mag["dx"] = res_scale * t, abs(res_scale) * tm
    if block is not None:
        b, g = np.asarray(block, np.float64), _gate(gate)
        du, dum = g * t, g * tm
        if w_post is not None:
            w, rb = np.asarray(w_post, np.float64), np.asarray(rstd_post, np.float64)[:, None]
            bh = b * rb
            u = w * bh
            r["dblock"] = rb * (w * du - bh * np.mean(w * du * bh, 1, keepdims=True))
            mag["dblock"] = rb * (np.abs(w) * dum + np.abs(bh) * np.mean(np.abs(w * bh) * dum, 1, keepdims=True))
            r["dw_post"], mag["dw_post"] = np.sum(du * bh, 0), np.sum(dum * np.abs(bh), 0)
        else:
            u = b
            r["dblock"], mag["dblock"] = du, dum
        if gate is not None:
            slope = g * _gate(gate, -1)
            dg, dgm = t * u * slope, tm * np.abs(u) * slope
            row = np.ndim(gate) == 1
            r["dgate"], mag["dgate"] = (dg.sum(1), dgm.sum(1)) if row else (dg, dgm)
    r["mag"] = mag
    return r


# ---------------------------------------------------------------------------------------------------- AdamW
def mix(x):
    """lowbias32."""
    x = np.asarray(x, np.uint64) & U32
    x = x ^ (x >> np.uint64(16))
    x = (x * np.uint64(0x7FEB352D)) & U32
    x = x ^ (x >> np.uint64(15))
    x = (x * np.uint64(0x846CA68B)) & U32
    return x ^ (x >> np.uint64(16))


def noise(n, seed, step, place=0):
    i = np.arange(place, place + n, dtype=np.uint64)
    key = mix(mix(np.uint64(seed)) ^ np.uint64(step & 0xFFFFFFFF))
    return mix((i & U32) ^ key ^ (((i >> np.uint64(32)) * np.uint64(0x9E3779B9)) & U32))


def _pow2(e):
    return np.ldexp(np.float32(1), np.asarray(e, np.int64) - 127).astype(np.float32)


def _blocks(x):
    pad = -x.size % BLOCK
    return np.concatenate([x, np.zeros(pad, x.dtype)]).reshape(-1, BLOCK)


def encode(x, u, second):
    """Codes and exponents of an fp32 array; u: noise of 19 (second moment) or 20 bits for every element."""
    drop = 19 if second else 20
    n = x.size
    a = _blocks(np.abs(np.asarray(x, np.float32)))
    e = np.minimum((a.max(1).view(np.uint32).astype(np.int64) + (1 << drop)) >> 23, 255)
    bad = ~np.isfinite(a).all(1)
    e[bad] = 255
    with np.errstate(invalid="ignore", over="ignore"):
        small = (a * _pow2(254 - np.minimum(e, 254))[:, None]) * np.float32(2.0 ** -112)
    code = (small.astype(np.float32).view(np.uint32).astype(np.int64) + _blocks(np.asarray(u, np.int64))) >> drop
    code[(e == 0) | (e == 255)] = 0
    if not second:
        code |= np.where(np.signbit(_blocks(np.asarray(x, np.float32))), 128, 0)
    return code.reshape(-1)[:n].astype(np.uint8), e.astype(np.uint8)


def decode(code, e, second):
    drop = 19 if second else 20
    n = code.size
    c = _blocks(np.asarray(code, np.uint8)).astype(np.uint32)
    mag = ((c if second else c & 127) << np.uint32(drop)).astype(np.uint32).view(np.float32)
    unit = np.where(e == 255, np.float32(np.nan), _pow2(np.minimum(e, 254).astype(np.int64)))[:, None]
    x = (mag * np.float32(2.0 ** 112)) * unit
    if not second:
        x = np.where(c > 127, -x, x)
    return x.reshape(-1)[:n].astype(np.float32)


def adamw(p, g, m, v, *, lr, betas, eps, weight_decay, step, coef=1.0):
    """(p, m, v) after a step, fp64."""
    p, g, m, v = (np.asarray(a, np.float64) for a in (p, g, m, v))
    b1, b2 = betas
    g = g * coef
    m, v = b1 * m + (1 - b1) * g, b2 * v + (1 - b2) * g * g
    upd = (m / (1 - b1 ** step)) / (np.sqrt(v / (1 - b2 ** step)) + eps)
    return p - lr * (weight_decay * p + upd), m, v


def adamw_states_8bit(g, m, m_exp, v, v_exp, *, betas, step, seed, coef=1.0, place=0):
    """The 8-bit moments after a step (m, m_exp, v, v_exp), in the fp32 operations that define them."""
    f = np.float32
    b1, b2 = betas
    g = np.asarray(g, f) * f(coef)
    m1 = decode(m, m_exp, False) * f(b1) + g * f(1 - b1)
    v1 = decode(v, v_exp, True) * f(b2) + (g * f(1 - b2)) * g
    u = noise(g.size, seed, step, place).astype(np.int64)
    vc, ve = encode(v1, u >> 13, True)
    mc, me = encode(m1, (u & 0xFFFF) << 4, False)
    mc[vc == 0] = 0
    return mc, me, vc, ve
