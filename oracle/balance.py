"""Plain float64 CPU oracle of the router's balance loss and its gradient.

TEST INFRASTRUCTURE ONLY, as oracle/moe.py.

For a sequence s with T_s live tokens, f_se = E / (k T_s) c_se over its live
tokens' top-k slots, P_se the mean of its live tokens' probabilities, and
loss = coef / S' sum_s sum_e f_se P_se over the S' sequences with a live token.
The counts are constants of the gradient.
"""

from __future__ import annotations

import numpy as np

__all__ = ["probabilities", "counts_of", "loss_given_counts", "loss", "gradient"]


def probabilities(logits):
    """softmax of each row; zeros where every logit is minus infinity."""
    x = np.asarray(logits, np.float64)
    out = np.zeros_like(x)
    for t in range(x.shape[0]):
        m = x[t].max()
        if m == -np.inf:
            continue
        e = np.exp(x[t] - m)
        out[t] = e / e.sum()
    return out


def _members(T, mask, seq, s):
    lo, hi = (0, T) if seq is None else (int(seq[s]), int(seq[s + 1]))
    return [t for t in range(lo, hi) if mask is None or mask[t]]


def counts_of(idx, mask, seq, S, T, E):
    """(counts [S, E], live [S + 1])"""
    counts, live = np.zeros((S, E), np.int32), np.zeros(S + 1, np.int32)
    for s in range(S):
        for t in _members(T, mask, seq, s):
            live[s] += 1
            for e in idx[t]:
                if 0 <= e < E:
                    counts[s, e] += 1
    live[S] = (live[:S] > 0).sum()
    return counts, live


def loss_given_counts(logits, counts, live, mask, seq, S, k, coef):
    T, E = logits.shape
    p = probabilities(logits)
    total = 0.0
    for s in range(S):
        t = _members(T, mask, seq, s)
        if t:
            total += float((counts[s] * E / (k * len(t)) * p[t].mean(axis=0)).sum())
    return coef * total / live[S] if live[S] else 0.0


def loss(logits, idx, mask, seq, S, coef):
    counts, live = counts_of(idx, mask, seq, S, *logits.shape)
    return loss_given_counts(logits, counts, live, mask, seq, S, idx.shape[1], coef), counts, live


def gradient(logits, counts, live, mask, seq, S, k, coef):
    T, E = logits.shape
    p = probabilities(logits)
    d = np.zeros((T, E))
    for s in range(S):
        t = _members(T, mask, seq, s)
        if t:
            f = counts[s] * E / (k * len(t))
            d[t] = coef / (live[S] * len(t)) * p[t] * (f[None, :] - (p[t] @ f)[:, None])
    return d
