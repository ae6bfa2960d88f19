"""Pins of the cache and attention oracle (no GPU)."""
from fractions import Fraction

import numpy as np
import pytest

from oracle import kv_oracle as kv


def test_quantise_by_hand():
    codes, s = kv.quantise(np.array([[127.0, -63.5, 0.5, 1.5, -2.5, 0.0, 126.5, -127.0]], np.float32))
    assert s.tolist() == [1.0]
    assert codes.tolist() == [[127, -64, 0, 2, -2, 0, 126, -127]]   # ties to even


def test_quantise_extremes():
    x = np.array([[0, 0], [2.0 ** -101, 0], [2.0 ** -100, 0], [np.nan, 1], [np.inf, 1], [-np.inf, np.nan], [3e38, -3e38]], np.float32)
    codes, s = kv.quantise(x)
    assert s[0] == 0 and s[1] == 0 and s[2] > 0 and np.isnan(s[3:6]).all() and np.isfinite(s[6])
    assert codes.tolist() == [[0, 0], [0, 0], [127, 0], [0, 0], [0, 0], [0, 0], [127, -127]]


def test_quantise_steps_are_the_rounded_rationals():
    rng = np.random.default_rng(0)
    x = rng.standard_normal((64, 16)).astype(np.float32)
    codes, s = kv.quantise(x)
    for row, c, si in zip(x, codes, s):
        a = Fraction(float(np.abs(row).max()))
        assert si == np.float32(float(a / 127))
        r = Fraction(float(np.float32(float(127 / a))))
        for xi, ci in zip(row, c):
            y = Fraction(float(np.float32(float(Fraction(float(xi)) * r))))
            assert ci == round(y)    # Fraction rounds half to even


def test_bf16_rounding():
    for x, want in [(1.0, 1.0), (1 + 2.0 ** -8, 1.0), (1 + 3 * 2.0 ** -8, 1 + 2.0 ** -6), (-1 - 2.0 ** -8 - 2.0 ** -20, -1 - 2.0 ** -7),
                    (3.4e38, np.inf), (np.inf, np.inf)]:
        assert kv.round_bf16(np.array([x]))[0] == want
    assert np.isnan(kv.round_bf16(np.array([np.nan]))[0])


@pytest.mark.parametrize("window,sinks", [(0, 0), (0, 2), (1, 0), (3, 0), (3, 2), (100, 1)])
def test_sees_by_enumeration(window, sinks):
    for p in range(-2, 9):
        want = [t for t in range(10) if t <= p and (window == 0 or p - window < t or t < sinks)]
        assert np.flatnonzero(kv.sees(p, np.arange(10), window, sinks)).tolist() == want


def test_attend_against_a_dense_softmax():
    rng = np.random.default_rng(1)
    page, D, H, G = 4, 8, 2, 3
    lens, offsets = np.array([9, 0, 5]), np.array([0, 4, 4, 9])
    table = np.array([[5, 1, 3], [9, 9, 9], [0, 4, -7]])
    kp, vp = rng.standard_normal((6, H, page, D)), rng.standard_normal((6, H, page, D))
    q = rng.standard_normal((9, H * G, D))
    out, lse, weight, spread = kv.attend(q, kp, vp, None, None, table, lens, offsets, 0.4)
    for b, (r0, n, L) in enumerate([(0, 4, 9), (4, 0, 0), (4, 5, 5)]):
        k = np.concatenate([kp[table[b, t // page], :, t % page][None] for t in range(L)]) if L else np.zeros((0, H, D))
        v = np.concatenate([vp[table[b, t // page], :, t % page][None] for t in range(L)]) if L else np.zeros((0, H, D))
        for i in range(n):
            for h in range(H * G):
                e = np.array([np.exp(0.4 * np.dot(q[r0 + i, h], k[t, h // G])) for t in range(L - n + i + 1)])
                want = sum(e[t] * v[t, h // G] for t in range(len(e))) / e.sum()
                assert np.allclose(out[r0 + i, h], want, rtol=1e-12, atol=1e-14)
                assert np.isclose(lse[r0 + i, h], np.log(e.sum()), rtol=1e-12)
                assert (weight[r0 + i, h] >= np.abs(out[r0 + i, h]) - 1e-12).all()


def test_rows_before_the_first_token_see_nothing():
    q = np.ones((4, 1, 2))
    out, lse, _, _ = kv.attend(q, np.ones((1, 1, 4, 2)), np.ones((1, 1, 4, 2)), None, None, np.array([[0]]), [2], [0, 4], 1.0)
    assert (out[:2] == 0).all() and (lse[:2] == -np.inf).all() and np.allclose(out[2:], 1)


def test_write_then_read():
    rng = np.random.default_rng(2)
    pool, scales = np.zeros((5, 2, 4, 8), np.int8), np.zeros((5, 2, 4), np.float32)
    table, lens, offsets = np.array([[3, 0], [7, 2]]), [6, 7], [0, 3, 6]
    x = rng.standard_normal((6, 2, 8))
    kv.write(pool, scales, kv.KV_I8, table, lens, offsets, x)
    got, written = kv.read(pool, scales, table, lens, offsets, 6)
    assert written.all()
    # the second sequence's first row (t = 4 .. 6) is on page 2; nothing of it is on the bad page 7
    assert np.abs(got - x).max() <= np.abs(x).max() / 127 / 2 + 1e-6
    assert (pool[[1, 4]] == 0).all()
