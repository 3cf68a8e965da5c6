"""Attention over caches that are read in full, and eviction, in float64 numpy.

Straight from the definitions, one query, head or slot at a time: a sliding
window with sinks, a shared prefix, accumulated weights, and the insertion into
a bounded cache that evicts by them.  Test infrastructure only.
"""
from __future__ import annotations

import math

import numpy as np


def attend(q, k, v, scale):
    """One query [d] over rows k, v [n][d]: (output, log-sum-exp, weights).  No
    rows, or logits of nothing but -inf: 0, -inf and weights of 0."""
    n = k.shape[0]
    if n == 0:
        return np.zeros(v.shape[1]), -math.inf, np.zeros(0)
    s = scale * (k @ q)
    m = s.max()
    if m == -math.inf:
        return np.zeros(v.shape[1]), -math.inf, np.zeros(n)
    e = np.exp(s - m)
    return (e / e.sum()) @ v, m + math.log(e.sum()), e / e.sum()


def visible(p, window, n_sink):
    """Tokens that a query at position p sees, ascending."""
    return [t for t in range(p + 1) if t < n_sink or t > p - window]


def window_attention(q, k, v, first, window, n_sink, scale):
    """q [T][H_q][d] at positions first, first + 1, ..; k, v [L][H_kv][d]:
    out [T][H_q][d], lse [T][H_q] and sum_t p |v| (what a relative error of the
    weights is multiplied by)."""
    T, H_q, d = q.shape
    G = H_q // k.shape[1]
    out, spread = np.zeros((T, H_q, d)), np.zeros((T, H_q, d))
    lse = np.full((T, H_q), -math.inf)
    for i in range(T):
        t = visible(first + i, window, n_sink)
        for h in range(H_q):
            kk, vv = k[t, h // G], v[t, h // G]
            out[i, h], lse[i, h], p = attend(q[i, h], kk, vv, scale)
            spread[i, h] = p @ np.abs(vv) if len(t) else 0.0
    return out, lse, spread


def prefix_attention(q, k_prefix, v_prefix, k, v, scale):
    """q [H_q][d] over the prefix rows [P][H_kv][d] followed by k, v [L][H_kv][d]."""
    H_q, d = q.shape
    G = H_q // k.shape[1]
    out, lse = np.zeros((H_q, d)), np.zeros(H_q)
    for h in range(H_q):
        out[h], lse[h], _ = attend(q[h], np.concatenate([k_prefix[:, h // G], k[:, h // G]]),
                                   np.concatenate([v_prefix[:, h // G], v[:, h // G]]), scale)
    return out, lse


def accumulate(q, k, v, n_sets, scale):
    """q [H_q][d] over k, v [L][H_kv][d]: out, lse and the weights added to each
    set's tokens [n_sets][L]."""
    H_q, d = q.shape
    G = H_q // k.shape[1]
    out, lse, w = np.zeros((H_q, d)), np.zeros(H_q), np.zeros((n_sets, k.shape[0]))
    for h in range(H_q):
        out[h], lse[h], p = attend(q[h], k[:, h // G], v[:, h // G], scale)
        w[h * n_sets // H_q] += p
    return out, lse, w


def evict_plan(weights, tokens, count, n_new, keep, pos, n_recent, n_sink):
    """One set: (rows held afterwards, [(slot, source)]) where a source is ('held',
    slot) or ('new', row)."""
    after = min(keep, count + n_new)
    taken = min(n_new, after)

    def rank(j):
        if tokens[j] < n_sink or tokens[j] >= pos + n_new - n_recent:
            w = math.inf
        elif math.isnan(weights[j]):
            w = -math.inf
        else:
            w = float(weights[j])
        return (-w, j)

    kept = sorted(sorted(range(count), key=rank)[:after - taken])
    free = [j for j in range(after) if j not in set(kept)]
    sources = [("held", j) for j in kept if j >= after]
    sources += [("new", i) for i in range(n_new - taken, n_new)]
    assert len(free) == len(sources)
    return after, list(zip(free, sources))
