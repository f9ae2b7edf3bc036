"""Oracle for the operators on rows of logits (float64 numpy) -- TEST INFRASTRUCTURE ONLY.

Row by row, from the definitions: tokens ranked by logit, then by id; the tokens that
stay under a temperature, top-k, top-p and min-p; inverse sampling in the order of the
ids; the divergence from a teacher's top logits and its gradient.  Each choice comes
with its margin: how far the nearest border is, relative to the mass it cuts, so that a
test can tell a wrong choice from a tie of two roundings.
"""
import numpy as np


def ranked(row):
    """Ids in the order of the row; a NaN counts as -inf, -0 equals 0."""
    x = np.where(np.isnan(row), -np.inf, np.asarray(row, np.float64)) + 0.0
    return x, np.argsort(-x, kind="stable")


def top(row, k):
    x, order = ranked(row)
    live = x[x > -np.inf]
    if not len(live):
        lse = -np.inf
    elif np.isinf(live.max()):
        lse = np.inf
    else:
        lse = live.max() + np.log(np.exp(live - live.max()).sum())
    return x[order[:k]], order[:k], lse


def weights(x, temperature):
    m = x.max()
    with np.errstate(invalid="ignore"):
        w = np.exp((x - m) / temperature)
    return np.where(x == m, 1.0, w)


def stay(row, temperature=1.0, top_k=0, top_p=1.0, min_p=0.0):
    """(ids that stay in ranked order, their weights, the margin of the choice)."""
    x, order = ranked(row)
    n = int((x > -np.inf).sum())
    if n == 0:
        return order[:0], np.zeros(0), np.inf
    if temperature == 0:
        temperature, top_k = 1.0, 1
    order = order[:n]
    w = weights(x[order], temperature)
    margin = np.inf
    if top_k:
        n = min(n, top_k)
    w = w[:n]
    if top_p < 1:
        mass = np.cumsum(w)
        border = top_p * mass[-1]
        margin = min(margin, float(np.abs(mass - border).min() / mass[-1]))
        n = min(n, int((mass < border).sum()) + 1)
    if min_p > 0:
        margin = min(margin, float(np.abs(w[1:] / min_p - 1).min(initial=np.inf)))
        n = min(n, max(1, int((w >= min_p).sum())))
    return order[:n], w[:n], margin


def sample(row, u, **how):
    """(token, log-probability, margin)."""
    ids, w, margin = stay(row, **how)
    if not len(ids):
        return -1, -np.inf, margin
    by_id = np.argsort(ids)
    mass = np.cumsum(w[by_id])
    at = min(max(float(u), 0.0), 1.0) * mass[-1] if u == u else 0.0
    i = min(int((mass <= at).sum()), len(ids) - 1)
    while w[by_id[i]] == 0:
        i -= 1
    margin = min(margin, float(np.abs(mass[:-1] - at).min(initial=np.inf) / mass[-1]))
    return int(ids[by_id[i]]), float(np.log(w[by_id[i]] / w.sum())), margin


def distill(row, ids, values, temperature, grad=1.0):
    """(loss, lse, gradient, p, q by id) of one row of a student."""
    x = np.asarray(row, np.float64) / temperature
    ids, t = np.asarray(ids), np.asarray(values, np.float64) / temperature
    here = (ids >= 0) & (ids < len(x))
    ids, t = ids[here], t[here]
    with np.errstate(invalid="ignore", divide="ignore"):
        m = np.max(x)
        lse = m + np.log(np.exp(x - m).sum()) if m != -np.inf else m
        p = np.exp(x - lse)
        q = np.zeros(len(x))
        if not len(t) or np.max(t) == -np.inf:
            return 0.0, lse, np.zeros(len(x)), p, q
        tm = np.max(t)
        e = np.exp(t - tm)
        np.add.at(q, ids, e / e.sum())
        lq = t - tm - np.log(e.sum())
        qi = e / e.sum()
        loss = np.where(qi == 0, 0.0, qi * (lq - (x[ids] - lse))).sum()
        if np.isnan(q).any():
            p = np.full(len(x), np.nan)
        return loss, lse, grad / temperature * (p - q), p, q
