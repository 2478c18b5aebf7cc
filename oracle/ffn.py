"""Plain float64 CPU oracle of the gated feed-forward block and its backward pass.

TEST INFRASTRUCTURE ONLY, as oracle/moe.py.

For rows in groups (offsets), with W1, W3 the first and last I rows of a group's
w_gate_up and W2 its w_down: g = x W1^T, u = x W3^T, h = silu(g) u, y = h W2^T, and
the gradients of a scalar whose gradient in y is dy.  Every function returns its
result and, where it sums products, the sums of their magnitudes, which bound what
rounding can do.
"""

from __future__ import annotations

import numpy as np

__all__ = ["sigmoid", "silu", "groups_of", "rows_times", "outer", "swiglu", "swiglu_gradient"]


def sigmoid(g):
    g = np.asarray(g, np.float64)
    with np.errstate(over="ignore"):
        return np.where(g >= 0, 1.0 / (1.0 + np.exp(-np.abs(g))), np.exp(-np.abs(g)) / (1.0 + np.exp(-np.abs(g))))


def silu(g):
    return np.asarray(g, np.float64) * sigmoid(g)


def groups_of(offsets, rows):
    """[(first row, one past the last)] of each group, clamped to [0, rows]."""
    if offsets is None:
        return [(0, rows)]
    o = np.clip(np.asarray(offsets, np.int64), 0, rows)
    return [(int(a), max(int(a), int(b))) for a, b in zip(o[:-1], o[1:])]


def rows_times(a, w, spans, transposed=True):
    """(each row times its group's matrix (its transpose), sums of magnitudes); NaN for rows of no group."""
    a, w = np.asarray(a, np.float64), np.asarray(w, np.float64)
    n = w.shape[1] if transposed else w.shape[2]
    out, mag = np.full((a.shape[0], n), np.nan), np.full((a.shape[0], n), np.nan)
    for e, (lo, hi) in enumerate(spans):
        m = w[e].T if transposed else w[e]
        out[lo:hi] = a[lo:hi] @ m
        mag[lo:hi] = np.abs(a[lo:hi]) @ np.abs(m)
    return out, mag


def outer(a, b, spans):
    """(each group's a^T b, sums of magnitudes)."""
    a, b = np.asarray(a, np.float64), np.asarray(b, np.float64)
    out = [a[lo:hi].T @ b[lo:hi] for lo, hi in spans]
    mag = [np.abs(a[lo:hi]).T @ np.abs(b[lo:hi]) for lo, hi in spans]
    return np.stack(out), np.stack(mag)


def swiglu(g, u):
    return silu(g) * np.asarray(u, np.float64)


def swiglu_gradient(g, u, dh):
    """(dg, du)"""
    s, t = sigmoid(g), sigmoid(-np.asarray(g, np.float64))
    return dh * u * s * (1.0 + np.asarray(g, np.float64) * t), dh * silu(g)
