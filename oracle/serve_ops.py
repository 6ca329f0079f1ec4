"""fp64 restatement of the operators of the base model's pass over a draft (test infrastructure only): attention over a paged
cache, eviction by accumulated attention weight, sampling from logits.  Plain loops over the definitions."""
from __future__ import annotations

import numpy as np


def places(table_row, page_slots: int, n: int):
    """(page, slot within it) of the first n slots of a sequence."""
    i = np.arange(n)
    return np.asarray(table_row)[i // page_slots], i % page_slots


def attend(q, K, V, fresh: int, scale: float) -> dict:
    """One sequence: q [Q, Hq, D], K and V [n, H, D]; the last `fresh` of the n slots are q's own first `fresh` rows.
    Returns out [fresh, Hq, D], lse [fresh, Hq], weights [H, n], and for error bounds `mass` = sum_i p_i |v_i| and
    `terms` = the largest scale * sum_d |q_d k_id| of a row."""
    n, H, D = K.shape
    Hq = q.shape[1]
    G = Hq // H
    out, mass = np.zeros((fresh, Hq, D)), np.zeros((fresh, Hq, D))
    lse, terms, weights = np.full((fresh, Hq), -np.inf), np.zeros((fresh, Hq)), np.zeros((H, n))
    for j in range(fresh):
        seen = n - (fresh - 1 - j)
        if seen <= 0:
            continue
        for h in range(Hq):
            k, v = K[:seen, h // G], V[:seen, h // G]
            s = k @ q[j, h] * scale
            terms[j, h] = abs(scale) * (np.abs(k) @ np.abs(q[j, h])).max()
            m = s.max()
            e = np.exp(s - m)
            p = e / e.sum()
            lse[j, h] = m + np.log(e.sum())
            out[j, h], mass[j, h] = p @ v, p @ np.abs(v)
            weights[h // G, :seen] += p
    return dict(out=out, lse=lse, weights=weights, mass=mass, terms=terms)


def evict(acc, n: int, budget: int, recent: int):
    """Kept slots of one head, in their order: acc [n]."""
    if n <= budget:
        return np.arange(n)
    key = np.where(np.isnan(acc), -np.inf, acc.astype(np.float64))
    old = n - recent
    order = np.lexsort((np.arange(old), -key[:old]))        # largest weight first, of equals the lowest slot
    # (NaN after -infinity's equals: both are the least)
    return np.sort(np.concatenate([order[:budget - recent], np.arange(old, n)])).astype(np.int64)


def sample(x, u: float, T: float, top_k: int, top_p: float, min_p: float) -> dict:
    """One row of logits [V]: the token, its log-probability, the number of entries kept, log-probabilities of all entries, and the
    distances of the decisions from their borders (relative to the masses that they compare)."""
    x = np.where(np.isnan(x), -np.inf, np.asarray(x, np.float64))
    V = x.shape[0]
    logp = np.full(V, -np.inf)
    if not (x > -np.inf).any():
        return dict(token=-1, logp=-np.inf, kept=0, all=logp, gap=np.inf)
    m = x.max()
    order = np.lexsort((np.arange(V), -x))
    order = order[x[order] > -np.inf]
    gap = np.inf
    if not T > 0:
        order, z = order[:1], np.zeros(V)
    else:
        if top_k > 0:
            order = order[:top_k]
        with np.errstate(invalid="ignore"):
            z = np.where(x == m, 0.0, (x - m) / T)
        if top_p < 1:
            c = np.cumsum(np.exp(z[order]))
            n = min(int((c < top_p * c[-1]).sum()) + 1, len(order))
            gap = np.abs(c / c[-1] - top_p).min()
            order = order[:n]
        if min_p > 0:
            w = np.exp(z[order])
            below = w[z[order] != 0]                           # (a weight of one is exact on both sides)
            gap = min(gap, np.abs(below / min_p - 1).min()) if len(below) else gap
            order = np.concatenate([order[:1], order[1:][w[1:] >= min_p]])
    keep = np.zeros(V, bool)
    keep[order] = True
    w = np.where(keep, np.exp(z), 0.0)
    run = np.cumsum(w)
    logp[keep] = z[keep] - np.log(run[-1])
    over = np.nonzero((run > u * run[-1]) & (w > 0))[0]
    token = int(over[0]) if len(over) else int(np.nonzero(w > 0)[0][-1])
    gap = min(gap, np.abs(run[keep] / run[-1] - u).min())
    return dict(token=token, logp=logp[token], kept=int(keep.sum()), all=logp, gap=gap)
