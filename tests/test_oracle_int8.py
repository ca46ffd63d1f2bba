"""Pins of the int8 oracle (oracle/int8.py)."""

from fractions import Fraction

import numpy as np

from oracle import bf16, int8


def _rows(seed, R=40, C=64):
    g = np.random.default_rng(seed)
    return bf16.to_f32(bf16.from_f64_rne(g.standard_t(3, (R, C)) * np.exp(g.normal(size=(R, 1)) * 8))).astype(np.float64)


def test_codes_are_the_nearest_integers_to_the_exact_product():
    x = _rows(1)
    q, s = int8.encode_rows(x)
    for i in range(len(x)):
        amax = np.abs(x[i]).max()
        r = Fraction(float(np.float32(np.float64(127) / amax)))
        assert s[i] == np.float32(amax / 127)
        for v, c in zip(x[i], q[i]):
            assert c == round(Fraction(float(v)) * r)             # (Fraction rounds ties to even)
    assert np.abs(q).max() == 127 and (np.abs(q).max(axis=1) == 127).all()


def test_factor_is_the_correctly_rounded_quotient():
    a = np.concatenate([np.random.default_rng(2).uniform(0.5, 2, 2000).astype(np.float32),
                        bf16.to_f32(np.arange(0x3F00, 0x4000, dtype=np.uint16))]).astype(np.float64)
    for v, r in zip(a, int8.factor(a)):
        exact = Fraction(127) / Fraction(float(v))
        near = [np.float32(r), np.nextafter(np.float32(r), np.float32(0)), np.nextafter(np.float32(r), np.float32(1e9))]
        assert min(abs(Fraction(float(n)) - exact) for n in near) == abs(Fraction(float(r)) - exact)


def test_special_rows():
    x = np.zeros((5, 16))
    x[1, 3], x[2, 5], x[3, :2] = np.inf, np.nan, (2.0 ** -133, -3 * 2.0 ** -133)
    x[4, :2] = 3.3895313892515355e38, -1.0
    q, s = int8.encode_rows(x)
    assert s[0] == 1 and not q[0].any() and np.isnan(s[1:3]).all() and not q[1:3].any()
    assert list(q[3, :3]) == [42, -127, 0] and q[4, 0] == 127 and q[4, 1] == 0


def test_transposed_copy_is_padded_with_zeros():
    x = _rows(3, 21, 32)
    q, s = int8.encode_cols(x)
    qr, sr = int8.encode_rows(x.T)
    assert q.shape == (32, 32) and (q[:, :21] == qr).all() and not q[:, 21:].any() and (s == sr).all()


def test_values_are_within_half_a_step():
    x = _rows(4)
    q, s = int8.encode_rows(x)
    assert (np.abs(q * s.astype(np.float64)[:, None] - x) <= s[:, None] * (0.5 + 1e-4)).all()


def test_bands_hold_the_exact_codes():
    x = _rows(5)
    lo, hi, s, tol = int8.band_rows(x, 2.0 ** -20)
    q, scale = int8.encode_rows(x)
    assert (lo <= q).all() and (q <= hi).all() and (hi - lo <= 1).all() and (np.abs(scale - s) <= tol).all()


def test_product_and_its_allowance():
    g = np.random.default_rng(6)
    A, B = g.integers(-127, 128, (5, 48)).astype(np.int8), g.integers(-127, 128, (7, 48)).astype(np.int8)
    sa, sb = g.random(5).astype(np.float32), g.random(7).astype(np.float32)
    d, tol = int8.gemm(A, sa, B, sb)
    for m in range(5):
        for n in range(7):
            acc = sum(int(a) * int(b) for a, b in zip(A[m], B[n]))
            f32 = np.float32(np.float32(acc) * sa[m]) * sb[n]
            assert abs(float(f32) - d[m, n]) <= tol[m, n]
            assert abs(d[m, n] - float(Fraction(acc) * Fraction(float(sa[m])) * Fraction(float(sb[n])))) <= 1e-15 * abs(d[m, n])
