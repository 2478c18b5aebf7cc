"""The oracles of the feed-forward block, the token rows and AdamW against differences, loops and hand-worked
values."""

import math

import numpy as np

from oracle import adamw as A
from oracle import ffn as F
from oracle import rows as R


def _block(x, wg, wu, wd):
    return F.swiglu(x @ wg.T, x @ wu.T) @ wd.T


def test_block_gradients_by_differences():
    rng = np.random.default_rng(0)
    H, I, rows = 5, 4, 3
    x, wg, wu, wd = rng.standard_normal((rows, H)), *(rng.standard_normal(s) for s in ((I, H), (I, H), (H, I)))
    c = rng.standard_normal((rows, H))  # the loss is sum(c y)
    g, u = x @ wg.T, x @ wu.T
    dh = c @ wd
    dg, du = F.swiglu_gradient(g, u, dh)
    got = [dg @ wg + du @ wu, dg.T @ x, du.T @ x, c.T @ F.swiglu(g, u)]
    for i, grad in enumerate(got):
        for at in np.ndindex(grad.shape):
            a = [x, wg, wu, wd]
            d = np.zeros_like(a[i])
            d[at] = 1e-6
            hi, lo = ((c * _block(*[v + s * d if j == i else v for j, v in enumerate(a)])).sum() for s in (1, -1))
            assert abs((hi - lo) / 2e-6 - grad[at]) < 1e-7 * max(1.0, abs(grad[at]))


def test_activation_far_out():
    g = np.array([-1e4, -800.0, -1.0, 0.0, 1.0, 800.0, 1e4])
    assert np.isfinite(F.sigmoid(g)).all() and F.silu(0.0) == 0
    assert F.sigmoid(1.0) + F.sigmoid(-1.0) == 1
    np.testing.assert_allclose(F.silu(g)[-2:], g[-2:])


def test_groups_and_products():
    assert F.groups_of(None, 7) == [(0, 7)]
    assert F.groups_of([-3, 2, 2, 9], 7) == [(0, 2), (2, 2), (2, 7)]
    a = np.arange(12.0).reshape(4, 3) - 5
    w = np.arange(12.0).reshape(2, 2, 3) - 4
    out, mag = F.rows_times(a, w, [(0, 1), (2, 4)])
    assert np.isnan(out[1]).all() and out[0, 0] == (a[0] * w[0, 0]).sum() and out[3, 1] == (a[3] * w[1, 1]).sum()
    assert mag[3, 1] == np.abs(a[3] * w[1, 1]).sum()
    dw, _ = F.outer(a, a, [(0, 1), (1, 1), (2, 4)])
    assert (dw[1] == 0).all() and dw[2, 1, 2] == a[2, 1] * a[2, 2] + a[3, 1] * a[3, 2]


def test_combine_gradients_by_differences():
    rng = np.random.default_rng(1)
    T, k, rows, H = 3, 2, 4, 3
    row = np.array([[0, 3], [-1, 2], [-1, 9]])
    y, w, c = rng.standard_normal((rows, H)), rng.standard_normal((T, k)), rng.standard_normal((T, H))
    dy, dw = R.combine_gradient(c, y, w, row, rows)
    loss = lambda y, w: (c * R.combine(y, w, row, rows)).sum()  # noqa: E731
    for at in np.ndindex(y.shape):
        d = np.zeros_like(y)
        d[at] = 1e-6
        want = dy[at[0]][at[1]] if at[0] in dy else 0.0
        assert abs((loss(y + d, w) - loss(y - d, w)) / 2e-6 - want) < 1e-8
    for at in np.ndindex(w.shape):
        d = np.zeros_like(w)
        d[at] = 1e-6
        assert abs((loss(y, w + d) - loss(y, w - d)) / 2e-6 - dw[at]) < 1e-8


def test_adamw_first_step():
    """At the first step from zero states the update is the gradient's sign, whatever its size."""
    p, m, v = A.step([1.0, 1.0], [3.0, -1e-3], [0, 0], [0, 0], 0.1, 1, 0.9, 0.99, 0.0, 0.5, 1.0)
    np.testing.assert_allclose(p, [1 - 0.1 * 1.5, 1 - 0.1 * (-1 + 0.5)])
    np.testing.assert_allclose(m, [0.3, -1e-4])
    np.testing.assert_allclose(v, [0.09, 1e-8])


def test_codes_by_hand():
    assert A.block_scale(0.0, 7) == 0 and A.block_scale(math.inf, 7) == 255
    assert A.block_scale(1.0, 0) == 127 and A.block_scale(1.99, 0) == 127 and A.block_scale(1.0, 7) == 120
    assert A.block_scale(2.0 ** -140, 0) == 0 and A.block_scale(3e38, 0) == 254
    # E4M3: 1 is exponent field 7, an eighth of it a mantissa step; below 2^-6 steps of 2^-9
    assert A.round_code(1.0, 0, -6) == 7 * 8 and A.round_code(1.125, 0, -6) == 7 * 8 + 1
    assert A.round_code(1.1, 0, -6) == 7 * 8 and A.round_code(1.1, 65535, -6) == 7 * 8 + 1
    assert A.round_code(1.99, 65535, -6) == 8 * 8  # carries into the next binade
    assert A.round_code(2.0 ** -9, 0, -6) == 1 and A.round_code(2.0 ** -9 * 0.5, 32767, -6) == 0
    assert A.round_code(2.0 ** -9 * 0.5, 32768, -6) == 1
    for code in range(0, 120):
        v = float(A.values_m(np.array([code]), np.array([127]))[0])
        assert A.round_code(v, 0, -6) == A.round_code(v, 65535, -6) == code  # a code's own value stays
    for code in range(256):
        v = float(A.values_root(np.array([code]), np.array([127]))[0])
        assert A.round_code(v, 0, -29) == A.round_code(v, 65535, -29) == code
    assert A.values_m(np.array([0x80 | 56]), np.array([130]))[0] == -8
    assert np.isnan(A.values_root(np.array([0]), np.array([255]))[0])


def test_words_are_spread():
    w = np.array(A.words(5, 17, 3, 4096))
    assert len(set(w.tolist())) == 4096  # a bijection of the place
    for half in (w >> 16, w & 0xFFFF):
        assert abs(half.mean() / 65535 - 0.5) < 6 / math.sqrt(12 * 4096)
    other = np.array(A.words(5, 18, 3, 4096))
    assert abs(np.corrcoef(w, other)[0, 1]) < 6 / 64
