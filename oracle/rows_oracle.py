"""Plain float64 oracle of the row operators (test infrastructure only): the top
entries of rows of logits, the distillation loss from such entries with its
gradient, and drawing a token under temperature, top-k, top-p and min-p.

Order of entries: value descending, then id ascending; NaN counts as -inf.
"""
from __future__ import annotations

import numpy as np


def _rows(logits):
    x = np.array(logits, dtype=np.float64)
    x[np.isnan(x)] = -np.inf
    return x


def _lse(x):
    """log(sum(exp(x))); -inf for nothing above -inf, +inf where there is one."""
    if x.size == 0:
        return -np.inf
    m = x.max()
    if np.isinf(m):
        return m
    return m + np.log(np.exp(x - m).sum())


def order(row):
    """Ids of a row in the order (value desc, id asc)."""
    return np.argsort(-row, kind="stable")


def top_logits(logits, k, temperature=1.0):
    x = _rows(logits)
    ids = np.stack([order(r)[:k] for r in x])
    vals = np.take_along_axis(x, ids, 1)
    rest = np.empty(len(x))
    for i, r in enumerate(x):
        others = np.ones(r.size, bool)
        others[ids[i]] = False
        rest[i] = _lse(r[others] / temperature)
    return dict(ids=ids.astype(np.int32), vals=vals, rest=rest)


def distill_row(row, ids, vals, rest, T):
    """(loss, gradient) of one row: loss T^2 KL over the entries' buckets and one of every other id."""
    V = row.size
    grad = np.zeros(V)
    used = ids >= 0
    ids, t = ids[used], np.where(np.isnan(vals[used]), -np.inf, vals[used])
    rest = -np.inf if np.isnan(rest) else rest
    if np.any(ids >= V) or len(set(ids.tolist())) < ids.size:
        return np.nan, np.full(V, np.nan)
    top = max(t, default=-np.inf)
    if max(top, rest) == -np.inf:
        return 0.0, grad
    if max(top, rest) == np.inf or row.max() == np.inf:  # no distribution
        return np.nan, np.full(V, np.nan)
    # relative to the larger of the first entry and the rest; differences first, t / T alone may be 1e38
    # (the rest's is of one product and one sum: 0 where it rounds past the other)
    t = np.append((t - top) / T, min(rest - top / T, 0.0)) if top / T >= rest else np.append(np.minimum(t / T - rest, 0.0), 0.0)
    log_p = t - _lse(t)
    p = np.exp(log_p)
    # (relative to the maximum: log(V) is lost beside values near the type's lowest)
    z = row / T if np.isinf(row.max()) else (row - row.max()) / T
    others = np.ones(V, bool)
    others[ids] = False
    lr, lz = _lse(z[others]), _lse(z)
    with np.errstate(invalid="ignore"):   # q = 0 wherever a logit (or all of them) is -inf
        log_q = np.where(np.append(z[ids], lr) == -np.inf, -np.inf, np.append(z[ids], lr) - lz)
    q = np.exp(log_q)
    some = p > 0
    loss = T * T * np.sum(p[some] * (log_p[some] - log_q[some]))
    grad[ids] = T * (q[:-1] - p[:-1])
    if lr > -np.inf:
        zo = z[others] - z[others].max()
        grad[others] = T * np.exp(zo - _lse(zo)) * (q[-1] - p[-1])
    return loss, grad


def distill_loss(logits, ids, vals, rest=None, temperature=1.0, weights=None, grad_scale=1.0):
    x = _rows(logits)
    n = len(x)
    T = float(temperature)
    w = np.ones(n) if weights is None else np.array(weights, np.float64)
    w[~(np.isfinite(w) & (w >= 0))] = 0.0
    rest = np.full(n, -np.inf) if rest is None else np.array(rest, np.float64)
    got = [distill_row(x[i], np.asarray(ids[i]), np.asarray(vals[i], np.float64), rest[i], T) for i in range(n)]
    row_loss = np.array([g[0] for g in got])
    W = w.sum()
    grad = np.zeros_like(x)
    loss = 0.0
    for i in np.flatnonzero(w > 0):
        loss += w[i] / W * row_loss[i]
        grad[i] = grad_scale * w[i] / W * got[i][1]
    return dict(loss=loss, row_loss=row_loss, grad=grad)


def sample_row(row, T=1.0, top_k=0, top_p=1.0, min_p=0.0, u=0.0):
    """(token, log-probability, kept entries, distance of u S from the nearest running sum over S)."""
    if row.max() == -np.inf:
        return -1, -np.inf, 0, 1.0
    ids = order(row)
    if T == 0:
        T, top_k = 1.0, 1
    x = row[ids]
    with np.errstate(invalid="ignore"):
        d = np.where(x == x[0], 0.0, (x[0] - x) / T)
    e = np.exp(-d)
    cum = np.cumsum(e)
    n_k = min(top_k, x.size) if top_k > 0 else x.size
    n = n_k
    if top_p < 1:
        n = min(n, max(1, int(np.sum(cum < top_p * cum[n_k - 1])) + 1))
    if min_p > 0:
        n = min(n, int(np.sum(e >= min_p)))
    S = cum[n - 1]
    i = min(int(np.sum(cum <= u * S)), n - 1)
    return int(ids[i]), -d[i] - np.log(S), n, float(np.min(np.abs(cum[:n] - u * S)) / S)


def sample_logits(logits, uniforms, temperature=None, top_k=None, top_p=None, min_p=None):
    x = _rows(logits)
    n = len(x)

    def of(a, i, default):
        return default if a is None else a[i]

    got = [sample_row(x[i], float(of(temperature, i, 1.0)), int(of(top_k, i, 0)), float(of(top_p, i, 1.0)),
                      float(of(min_p, i, 0.0)), float(uniforms[i])) for i in range(n)]
    return dict(tokens=np.array([g[0] for g in got], np.int32), logprobs=np.array([g[1] for g in got]),
                kept=np.array([g[2] for g in got]), margin=np.array([g[3] for g in got]))
