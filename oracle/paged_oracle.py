"""CPU oracle for the operators on a paged key/value cache (float64 NumPy).

TEST INFRASTRUCTURE ONLY (same rules as domino_oracle).  The definitions are those of
include/domino.h; the paper's serving numbers (Sec. 5) are taken behind a serving engine, whose
cache it does not describe, so parity is unpinned beyond them.  Caches are arrays
[layers, pages, page_size, n_kv, d_h], weights [layers, pages, n_kv, page_size], updated in place.
"""
from __future__ import annotations

import numpy as np

F64 = np.float64


def rope_frequencies(rot, theta, scaling="none", factor=1.0, original_ctx=0, beta_fast=32.0, beta_slow=1.0):
    """Angles a position of every rotated pair, and the factor on the rotated elements."""
    i = np.arange(rot // 2, dtype=F64)
    if scaling == "ntk":
        theta = theta * factor ** (rot / (rot - 2))
    f = F64(theta) ** (-2.0 * i / rot)
    if scaling == "linear":
        f = f / factor
    if scaling == "yarn":
        keep = np.clip((original_ctx * f / (2 * np.pi) - beta_slow) / (beta_fast - beta_slow), 0.0, 1.0)
        return f * keep + f / factor * (1 - keep), 0.1 * np.log(factor) + 1.0
    return f, 1.0


def rotate(x, pos, freq, scale=1.0, interleaved=False, gain=None, eps=1e-6):
    """[tokens, heads, d_h] heads, normalised with `gain`, their first 2 len(freq) elements rotated.  Also returns what
    an error relative to the operands is measured by: |x cos| + |y sin|."""
    x = np.asarray(x, F64)
    if gain is not None:
        x = x / np.sqrt((x * x).mean(-1, keepdims=True) + eps) * np.asarray(gain, F64)
    y, size = x.copy(), np.abs(x)
    n = len(freq)
    if n:
        a = np.asarray(pos, F64)[:, None, None] * freq
        c, s = np.cos(a) * scale, np.sin(a) * scale
        i, j = (slice(0, 2 * n, 2), slice(1, 2 * n, 2)) if interleaved else (slice(0, n), slice(n, 2 * n))
        y[..., i], y[..., j] = x[..., i] * c - x[..., j] * s, x[..., j] * c + x[..., i] * s
        size[..., i] = size[..., j] = np.abs(x[..., i]) * scale + np.abs(x[..., j]) * scale
    return y, size


def cells(table, b, slots, page):
    """(pages, rows in them) of a sequence's slots."""
    slots = np.asarray(slots)
    return np.asarray(table)[b, slots // page], slots % page


def gather(cache, table, b, n, layer, head):
    """A sequence's first n rows of one head, [n, d_h]."""
    p, r = cells(table, b, np.arange(n), cache.shape[2])
    return np.asarray(cache[layer, p, r, head], F64)


def attention(q, k_cache, v_cache, table, starts, lens, layer, scale, mask=None):
    """Outputs [tokens, n_q, d_h], lse [tokens, n_q], the weights that each sequence's slots receive ({(b, head): [len]}),
    and per row what bounds its errors: the largest sum |q||k| scale, and sum p |v|."""
    q = np.asarray(q, F64)
    nq, dh, nkv = q.shape[1], q.shape[2], k_cache.shape[3]
    out, lse = np.zeros_like(q), np.full(q.shape[:2], -np.inf)
    size, spread, given = np.zeros(q.shape[:2]), np.zeros_like(q), {}
    for b in range(len(lens)):
        lo, hi, n = starts[b], starts[b + 1], lens[b]
        if lo == hi:
            continue
        new = hi - lo
        seen = np.ones((new, n), bool)
        seen[:, n - new:] = np.tril(np.ones((new, new), bool)) if mask is None else np.asarray(mask[lo:hi, :new]) != 0
        for h in range(nkv):
            k, v = (gather(c, table, b, n, layer, h) for c in (k_cache, v_cache))
            total = np.zeros(n)
            for j in range(h * (nq // nkv), (h + 1) * (nq // nkv)):
                row = q[lo:hi, j]
                with np.errstate(invalid="ignore"):   # (a hidden slot may hold anything)
                    s = np.where(seen, row @ k.T * scale, -np.inf)
                    size[lo:hi, j] = np.where(seen, np.abs(row) @ np.abs(k).T * scale, 0).max(1)
                top = s.max(1, keepdims=True)
                live = top[:, 0] > -np.inf
                e = np.where(seen & live[:, None], np.exp(s - np.where(live[:, None], top, 0)), 0.0)
                p = e / np.maximum(e.sum(1, keepdims=True), 1e-300)
                for i in range(new):
                    vi = v[seen[i]]
                    out[lo + i, j], spread[lo + i, j] = p[i][seen[i]] @ vi, p[i][seen[i]] @ np.abs(vi)
                lse[lo:hi, j] = np.where(live, np.log(np.maximum(e.sum(1), 1e-300)) + np.where(live, top[:, 0], 0), -np.inf)
                total += p.sum(0)
            given[b, h] = total
    return out, lse, given, size, spread


def evict_choice(w, budget, sink, recent):
    """The slots of one head that stay, ascending."""
    n = len(w)
    if n <= budget:
        return np.arange(n)
    mid = np.arange(sink, n - recent)
    key = np.where(np.isnan(w[mid]), -np.inf, w[mid])
    rank = np.lexsort((mid, np.isnan(w[mid]), -key))
    return np.sort(np.concatenate([np.arange(sink), mid[rank[:budget - sink - recent]], np.arange(n - recent, n)]))


def evict(k, v, w, table, lens, budget, sink, recent, new_table=None):
    """Updates the caches; new lengths and the kept slots [layers, batch, n_kv, budget], -1 padded."""
    layers, _, page, nkv, _ = k.shape
    kept = np.full((layers, len(lens), nkv, budget), -1, np.int32)
    for b, n in enumerate(lens):
        p, r = cells(table, b, np.arange(n), page)
        for layer in range(layers):
            for h in range(nkv):
                s = evict_choice(w[layer, p, h, r], budget, sink, recent)
                kept[layer, b, h, :len(s)] = s
                if n <= budget and new_table is None:
                    continue
                to, at = cells(table if new_table is None else new_table, b, np.arange(len(s)), page)
                k[layer, to, at, h] = k[layer, p[s], r[s], h]
                v[layer, to, at, h] = v[layer, p[s], r[s], h]
                w[layer, to, h, at] = w[layer, p[s], h, r[s]]
    return np.minimum(lens, budget).astype(np.int32), kept


def commit(k, v, w, table, ctx_lens, accept_len, accepted):
    page = k.shape[2]
    for b, (n, a) in enumerate(zip(ctx_lens, accept_len)):
        if a == 0:
            continue
        p, r = cells(table, b, n + np.asarray(accepted[b][:a]), page)
        to, at = cells(table, b, n + 1 + np.arange(a), page)
        k[:, to, at] = k[:, p, r]
        v[:, to, at] = v[:, p, r]
        if w is not None:
            w[:, to, :, at] = w[:, p, :, r]
    return (np.asarray(ctx_lens) + 1 + np.asarray(accept_len)).astype(np.int32)
