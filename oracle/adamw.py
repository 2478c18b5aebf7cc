"""CPU oracle of an AdamW step with states in 32 bits or in 8.

TEST INFRASTRUCTURE ONLY, as oracle/moe.py.

The step itself in float64; the codes of 8-bit states from their definition, one
value at a time, given the float32 values that are rounded.
"""

from __future__ import annotations

import math

import numpy as np

__all__ = ["step", "states32", "mix", "words", "block_scale", "round_code", "codes", "values_m", "values_root"]


def step(p, g, m, v, lr, t, beta1, beta2, eps, decay, scale):
    """(p, m, v) after one step, in float64."""
    p, m, v = (np.asarray(a, np.float64) for a in (p, m, v))
    g = np.asarray(g, np.float64) * scale
    m = beta1 * m + (1 - beta1) * g
    v = beta2 * v + (1 - beta2) * g * g
    p = p - lr * (m / (1 - beta1 ** t) / (np.sqrt(v / (1 - beta2 ** t)) + eps) + decay * p)
    return p, m, v


def states32(g, m, v, beta1, beta2, scale):
    """m and v with each operation rounded to float32, in the formulas' order."""
    f = np.float32
    g = (np.asarray(g, f) * f(scale)).astype(f)
    m = (f(beta1) * np.asarray(m, f)).astype(f) + (f(1 - beta1) * g).astype(f)
    v = (f(beta2) * np.asarray(v, f)).astype(f) + ((f(1 - beta2) * g).astype(f) * g).astype(f)
    return m.astype(f), v.astype(f)


def mix(a):
    a ^= a >> 16
    a = a * 0x6A09E667 % 2 ** 32
    a ^= a >> 15
    a = a * 0xBB67AE85 % 2 ** 32
    return a ^ (a >> 16)


def words(seed, t, tensor, n):
    key = mix((mix((mix(seed) + t) % 2 ** 32) + tensor) % 2 ** 32)
    return [mix(i ^ key) for i in range(n)]


def block_scale(top, above):
    """The scale byte of a block whose largest magnitude is `top`: into [2^above, 2^(above + 1))."""
    if not math.isfinite(top):
        return 255
    if top == 0:
        return 0
    return min(254, max(0, math.frexp(top)[1] - 1 - above + 127))


def round_code(q, r, low):
    """The code of the magnitude q whose smallest normal number is 2^low, with r 2^-16 added before the cut."""
    e = max(math.frexp(q)[1] - 1, low) if q > 0 else low
    n = math.floor(q / 2.0 ** (e - 3) + r / 65536)  # 8 to 16 of the binade's steps, or fewer below
    return (e - low) * 8 + n


def codes(m, root, word):
    """(m's codes, m's scales, the root's codes, the root's scales) of float32 values."""
    n = len(m)
    mc, vc, ms, vs = np.zeros(n, np.uint8), np.zeros(n, np.uint8), [], []
    for b in range(0, n, 32):
        at = range(b, min(b + 32, n))
        nan = lambda a: any(not math.isfinite(float(a[i])) for i in at)  # noqa: E731
        S = block_scale(math.inf if nan(m) else max(abs(float(m[i])) for i in at), 7)
        R = block_scale(math.inf if nan(root) else max(abs(float(root[i])) for i in at), 0)
        ms.append(S)
        vs.append(R)
        for i in at:
            if S != 255:
                mc[i] = round_code(abs(float(m[i])) * 2.0 ** (127 - S), word[i] >> 16, -6) | (128 if m[i] < 0 else 0)
            if R != 255:
                c = round_code(float(root[i]) * 2.0 ** (127 - R), word[i] & 0xFFFF, -29)
                vc[i] = max(c, 1) if root[i] > 0 else c
    return mc, np.array(ms, np.uint8), vc, np.array(vs, np.uint8)


def _scaled(v, scales):
    s = np.asarray(scales, np.float64)[np.arange(len(v)) // 32]
    return np.where(s == 255, np.nan, v * 2.0 ** (s - 127))


def values_m(code, scales):
    c = np.asarray(code, np.int64)
    e, f = (c & 127) >> 3, c & 7
    v = np.where(e > 0, (1 + f / 8) * 2.0 ** (e - 7.0), f / 8 * 2.0 ** -6)
    return _scaled(np.where(c & 128, -v, v), scales)


def values_root(code, scales):
    c = np.asarray(code, np.int64)
    e, f = c >> 3, c & 7
    return _scaled(np.where(e > 0, (1 + f / 8) * 2.0 ** (e - 30.0), f / 8 * 2.0 ** -29), scales)
