"""Plain CPU oracle of the MX FP4 matrices and products: OCP microscaling with
E2M1 elements and a shared E8M0 scale per 32 consecutive values along K.

TEST INFRASTRUCTURE ONLY, as oracle/moe.py: nothing of the product imports it,
and it imports nothing from the product package.

* E2M1: 1 sign, 2 exponent bits with bias 1, 1 mantissa bit: magnitudes 0, 0.5,
  1, 1.5, 2, 3, 4, 6; no infinities, no NaN.
* A block's exponent is floor(log2(amax)) - 2 (2 is E2M1's largest exponent),
  clamped to [-127, 127], or -127 when amax = 0; each value becomes the code of
  v / 2^E rounded to nearest, ties to the even code, magnitudes above 6 to 6.  A
  block that holds a NaN or an infinity has scale 255 (E8M0's NaN).
* Products multiply the dequantized values in float64.
* hold / release: the order in which a matrix is kept on the device.
"""

from __future__ import annotations

import numpy as np

__all__ = ["e2m1_decode", "e2m1_encode", "quantize", "dequantize", "hold", "release", "product", "swiglu"]

BLOCK = 32
E2M1_MAX = 6.0
E2M1_EMAX = 2


def e2m1_decode(codes) -> np.ndarray:
    c = np.asarray(codes, np.uint8).astype(np.int64)
    e, m = (c >> 1) & 3, c & 1
    mag = np.where(e == 0, 0.5 * m, (1.0 + 0.5 * m) * np.exp2(e - 1.0))
    return np.where(c & 8, -mag, mag)


def e2m1_encode(v) -> np.ndarray:
    v = np.asarray(v, np.float64)
    a = np.minimum(np.abs(v), E2M1_MAX)
    # the spacing of codes is 0.5 below 2, 1 below 4, 2 above; codes count the
    # spacings, so rounding the count half to even rounds to the even code
    code = np.where(a < 2.0, np.round(a * 2.0), np.where(a < 4.0, 2.0 + np.round(a), 4.0 + np.round(a / 2.0)))
    return (code.astype(np.int64) | (np.signbit(v).astype(np.int64) << 3)).astype(np.uint8)


def quantize(v):
    """(codes [R, K], scale bytes [R, K / 32]) of rows of whole blocks."""
    v = np.asarray(v, np.float64)
    R, K = v.shape
    b = v.reshape(R, K // BLOCK, BLOCK)
    bad = ~np.isfinite(b).all(axis=2)
    b = np.where(bad[:, :, None], 0.0, b)
    amax = np.abs(b).max(axis=2)
    _, ex = np.frexp(amax)  # amax = m 2^ex, m in [0.5, 1): floor(log2 amax) = ex - 1
    e = np.where(amax > 0, np.clip(ex - 1 - E2M1_EMAX, -127, 127), -127)
    codes = e2m1_encode(b / np.exp2(e.astype(np.float64))[:, :, None]).reshape(R, K)
    codes = np.where(np.repeat(bad, BLOCK, axis=1), 0, codes).astype(np.uint8)
    return codes, np.where(bad, 255, e + 127).astype(np.uint8)


def dequantize(codes, scales) -> np.ndarray:
    codes = np.asarray(codes)
    s = np.asarray(scales).astype(np.float64)
    s = np.where(s == 255.0, np.nan, np.exp2(s - 127.0))
    return e2m1_decode(codes) * np.repeat(s, BLOCK, axis=1)


def _up(v, m):
    return -(-v // m) * m


def hold(codes, scales):
    """Row-major codes (one a byte) and scales of whole blocks -> the held bytes."""
    R, K = codes.shape
    Rp, Kp = _up(R, 32), _up(K, 256)
    c = np.zeros((Rp, Kp), np.uint8)
    c[:R, :K] = codes
    s = np.zeros((Rp, Kp // 32), np.uint8)
    s[:R, :K // 32] = scales
    held_c = np.zeros((Rp // 32, Kp // 32, 32, 16), np.uint8)
    held_s = np.zeros((Rp // 32, Kp // 256, 2, 32, 4), np.uint8)
    pairs = c[:, 0::2] | (c[:, 1::2] << 4)
    for b in range(Kp // 32):
        held_c[:, b] = pairs[:, 16 * b:16 * b + 16].reshape(Rp // 32, 32, 16)
        held_s[:, b // 8, b % 2, :, (b % 8) // 2] = s[:, b].reshape(Rp // 32, 32)
    return held_c.reshape(-1), held_s.reshape(-1)


def release(held_c, held_s, R, K):
    """The inverse of hold, for K padded to whole slices of 256."""
    Rp, Kp = _up(R, 32), _up(K, 256)
    held_c = np.asarray(held_c).reshape(Rp // 32, Kp // 32, 32, 16)
    held_s = np.asarray(held_s).reshape(Rp // 32, Kp // 256, 2, 32, 4)
    c = np.zeros((Rp, Kp), np.uint8)
    s = np.zeros((Rp, Kp // 32), np.uint8)
    for b in range(Kp // 32):
        pairs = held_c[:, b].reshape(Rp, 16)
        c[:, 32 * b:32 * b + 32:2] = pairs & 15
        c[:, 32 * b + 1:32 * b + 32:2] = pairs >> 4
        s[:, b] = held_s[:, b // 8, b % 2, :, (b % 8) // 2].reshape(Rp)
    return c[:R], s[:R]


def product(a, w, offsets, n):
    """(y, sum of |a w|): rows [offsets[g], offsets[g + 1]) of a times w[g n : (g + 1) n]^T;
    rows of no group are NaN."""
    y = np.full((a.shape[0], n), np.nan)
    mag = np.full((a.shape[0], n), np.nan)
    for g in range(len(offsets) - 1):
        lo, hi = int(offsets[g]), int(offsets[g + 1])
        if lo < hi:
            m = w[g * n:(g + 1) * n]
            y[lo:hi] = a[lo:hi] @ m.T
            mag[lo:hi] = np.abs(a[lo:hi]) @ np.abs(m).T
    return y, mag


def swiglu(gate, up):
    with np.errstate(over="ignore"):
        return gate / (1.0 + np.exp(-gate)) * up
