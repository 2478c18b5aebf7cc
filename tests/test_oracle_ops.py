"""Pins of the oracles of the MX FP4 matrices (oracle/mx4.py) and of the balance
loss (oracle/balance.py) against things other than themselves."""

import math

import numpy as np
import pytest

from oracle import balance as B
from oracle import mx4 as X

MAGNITUDES = [0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0]


def test_e2m1_codes_are_the_formats():
    assert X.e2m1_decode(np.arange(16)).tolist() == MAGNITUDES + [-v for v in MAGNITUDES]


def test_encode_is_the_nearest_code_ties_to_even():
    mids = [0.5 * (a + b) for a, b in zip(MAGNITUDES, MAGNITUDES[1:])]
    vals = MAGNITUDES + mids + [math.nextafter(m, 0) for m in mids] + [math.nextafter(m, 9) for m in mids] + [6.5, 7.99]
    for v in vals:
        dist = [abs(min(v, 6.0) - m) for m in MAGNITUDES]
        near = [i for i in range(8) if dist[i] == min(dist)]
        want = near[0] if len(near) == 1 else [i for i in near if i % 2 == 0][0]
        assert X.e2m1_encode([v])[0] == want, v
        assert X.e2m1_encode([-v])[0] == want | 8, v


def test_hand_worked_blocks():
    v = np.zeros((1, 160))
    v[0, :4] = [7.9, -6.0, 0.25, 0.2501]    # exponent 0: 7.9 clips to 6
    v[0, 32] = 2.0 ** -140                  # below the smallest exponent
    v[0, 64] = np.inf
    v[0, 96:98] = [1.0, 0.1]                # exponent -2: 4 and 0.4
    c, s = X.quantize(v)
    assert s[0].tolist() == [127, 0, 255, 125, 0]
    assert c[0, :4].tolist() == [7, 15, 0, 1] and c[0, 96:98].tolist() == [6, 1] and not c[0, 64:96].any()
    d = X.dequantize(c, s)
    assert d[0, :4].tolist() == [6.0, -6.0, 0.0, 0.5] and np.isnan(d[0, 64:96]).all()


def test_quantize_error_bound_and_hold_round_trip():
    rng = np.random.default_rng(3)
    v = rng.standard_normal((45, 320)) * np.exp2(rng.integers(-20, 20, (45, 1)))
    c, s = X.quantize(v)
    d = X.dequantize(c, s)
    amax = np.abs(v).reshape(45, 10, 32).max(axis=2).repeat(32, axis=1)
    # half the widest spacing, or the clip from 8 to 6, of exponent floor(log2 amax) - 2
    assert (np.abs(d - v) <= 0.25 * np.maximum(2.0 ** np.floor(np.log2(amax)), 0) * 2.0 + 1e-300).all()
    assert ((np.abs(d) > 0) | (np.abs(v) <= amax / 8)).all()
    hc, hs = X.hold(c, s)
    assert hc.size == 64 * 512 // 2 and hs.size == 64 * 512 // 32
    # one value's place, spelt out: row 37, column 300 = block 9, value 12
    assert (hc.reshape(2, 16, 32, 16)[1, 9, 5, 6] & 15) == c[37, 300]
    assert hs.reshape(2, 2, 2, 32, 4)[1, 1, 1, 5, 0] == s[37, 9]
    c2, s2 = X.release(hc, hs, 45, 320)
    assert np.array_equal(c2[:, :320], c) and np.array_equal(s2[:, :10], s) and not c2[:, 320:].any()


def test_product_is_the_triple_loop():
    rng = np.random.default_rng(4)
    a, w = rng.standard_normal((5, 7)), rng.standard_normal((6, 7))
    y, mag = X.product(a, w, [1, 3, 3, 4], 2)
    assert np.isnan(y[0]).all() and np.isnan(y[4]).all()
    for r, g in ((1, 0), (2, 0), (3, 2)):
        for c in range(2):
            t = [a[r, i] * w[2 * g + c, i] for i in range(7)]
            assert math.isclose(y[r, c], math.fsum(t), rel_tol=1e-13, abs_tol=1e-13)
            assert math.isclose(mag[r, c], math.fsum(map(abs, t)), rel_tol=1e-13)
    assert X.swiglu(np.array([2.0]), np.array([3.0]))[0] == pytest.approx(6.0 / (1 + math.exp(-2.0)), rel=1e-15)
    assert X.swiglu(np.array([-800.0]), np.array([3.0]))[0] == 0.0


def _example(seed=0, T=23, E=7, k=3, S=4):
    rng = np.random.default_rng(seed)
    logits = rng.standard_normal((T, E)) * 2
    idx = np.argsort(-logits, axis=1)[:, :k].astype(np.int32)
    mask = (rng.random(T) < 0.8).astype(np.uint8)
    seq = np.array([0, 5, 5, 6, T][:S + 1], np.int32)
    return logits, idx, mask, seq, S


def test_even_routing_gives_coef():
    E, k = 8, 2
    idx = np.array([[(2 * t) % E, (2 * t + 1) % E] for t in range(12)], np.int32)
    value, counts, live = B.loss(np.zeros((12, E)), idx, None, None, 1, 0.25)
    assert value == pytest.approx(0.25, rel=1e-15) and counts.tolist() == [[3] * 8] and live.tolist() == [12, 1]


def test_loss_by_hand():
    # one token, two experts, probability 3/4 on the chosen one: E / (k T) c P = 2 * 3/4
    value, _, _ = B.loss(np.array([[math.log(3.0), 0.0]]), np.array([[0]], np.int32), None, None, 1, 1.0)
    assert value == pytest.approx(1.5, rel=1e-15)


def test_gradient_is_that_of_differences():
    logits, idx, mask, seq, S = _example()
    k, coef, h = idx.shape[1], 0.7, 1e-6
    _, counts, live = B.loss(logits, idx, mask, seq, S, coef)
    d = B.gradient(logits, counts, live, mask, seq, S, k, coef)
    for t in range(logits.shape[0]):
        for e in range(logits.shape[1]):
            up, dn = logits.copy(), logits.copy()
            up[t, e] += h
            dn[t, e] -= h
            f = lambda x: B.loss_given_counts(x, counts, live, mask, seq, S, k, coef)
            assert (f(up) - f(dn)) / (2 * h) == pytest.approx(d[t, e], abs=1e-9)
    assert not d[mask == 0].any()
