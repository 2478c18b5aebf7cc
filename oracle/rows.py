"""Plain float64 CPU oracle of token rows there and back, and of the gate's gradient.

TEST INFRASTRUCTURE ONLY, as oracle/moe.py.
"""

from __future__ import annotations

import numpy as np

__all__ = ["combine", "combine_gradient", "gate_gradient"]


def combine(y, w, row_of_slot, rows):
    """out[t] = sum over the slots with a row of w y[row]; w None: 1."""
    T, k = row_of_slot.shape
    out = np.zeros((T, y.shape[1]))
    for t in range(T):
        for j in range(k):
            r = row_of_slot[t, j]
            if 0 <= r < rows:
                out[t] += (1.0 if w is None else float(w[t, j])) * y[r].astype(np.float64)
    return out


def combine_gradient(dout, y, w, row_of_slot, rows):
    """({row: dy}, dw)"""
    T, k = row_of_slot.shape
    dy, dw = {}, np.zeros((T, k))
    for t in range(T):
        for j in range(k):
            r = row_of_slot[t, j]
            if 0 <= r < rows:
                d = dout[t].astype(np.float64)
                dy[int(r)] = (1.0 if w is None else float(w[t, j])) * d
                dw[t, j] = (d * y[r].astype(np.float64)).sum()
    return dy, dw


def gate_gradient(idx, w, dw, E):
    """The gradient in the logits of weights that are softmaxes over the picked logits."""
    T, k = idx.shape
    out = np.zeros((T, E))
    w, dw = w.astype(np.float64), dw.astype(np.float64)
    for t in range(T):
        mean = (w[t] * dw[t]).sum()
        for j in range(k):
            if 0 <= idx[t, j] < E:
                out[t, idx[t, j]] += w[t, j] * (dw[t, j] - mean)
    return out
