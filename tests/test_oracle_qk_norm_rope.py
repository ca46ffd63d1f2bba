"""Pins of the query / key norm and rotation oracle (oracle/qk_norm_rope.py)."""

import numpy as np
import pytest

from oracle import bf16, qk_norm_rope as qk


def _case(seed, T=3, H=2, D=16, R=16):
    g = np.random.default_rng(seed)
    cos, sin = qk.angles(g.integers(0, 5000, T), R, 1e4)
    return g.normal(size=(T, H, D)), 1 + 0.3 * g.normal(size=D), cos, sin, g.normal(size=(T, H, D))


@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("R", [0, 6, 16])
def test_rotation_is_a_complex_product(R, interleaved):
    x, _, _, _, _ = _case(1)
    p = np.array([0, 7, 123456])
    cos, sin = qk.angles(p, R, 1e6)
    y, _ = qk.rotate(x, cos, sin, interleaved)
    head = x[..., :R]
    z = head[..., 0::2] + 1j * head[..., 1::2] if interleaved else head[..., :R // 2] + 1j * head[..., R // 2:]
    z = z * (cos + 1j * sin)[:, None, :]
    np.testing.assert_allclose(y[..., :R], np.stack((z.real, z.imag), -1).reshape(head.shape) if interleaved
                               else np.concatenate((z.real, z.imag), -1), atol=1e-15)
    assert (y[..., R:] == x[..., R:]).all()
    assert (y[0] == x[0]).all()                                  # position 0
    np.testing.assert_allclose((y * y).sum(-1), (x * x).sum(-1), rtol=1e-14)


def test_products_depend_on_the_distance():
    g = np.random.default_rng(2)
    q, k = g.normal(size=(1, 1, 32)), g.normal(size=(1, 1, 32))
    dots = []
    for p in (0, 11, 4000):
        (a, _), (b, _) = (qk.rotate(v, *qk.angles([at], 32, 1e4), False) for v, at in ((q, p), (k, p + 37)))
        dots.append((a * b).sum())
    np.testing.assert_allclose(dots, dots[0], rtol=1e-11)


def test_norm_closed_forms():
    x = np.full((1, 1, 8), -3.0)
    none = np.zeros((1, 0))
    np.testing.assert_allclose(qk.forward(x, np.full(8, 2.0), 0.0, none, none)[0], -2.0)
    y, _ = qk.forward(np.zeros((1, 1, 8)), np.ones(8), 1e-6, none, none)
    assert (y == 0).all()
    # eps dominates a tiny head: n = x / sqrt(eps)
    e = float(np.float32(1e-6))
    np.testing.assert_allclose(qk.forward(x * 2.0 ** -40, np.ones(8), 1e-6, none, none)[0], -3 * 2.0 ** -40 / e ** 0.5)
    assert (qk.forward(x, None, 1e-6, none, none)[0] == x).all()


@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("norm", [False, True])
@pytest.mark.parametrize("R", [0, 8, 16])
def test_backward_by_differences(R, norm, interleaved):
    x, gamma, _, _, dy = _case(3)
    cos, sin = qk.angles([1, 50, 4097], R, 1e4)
    gamma = gamma if norm else None
    dx, _, dgamma, _ = qk.backward(dy, x, gamma, 1e-6, cos, sin, interleaved)
    f = lambda x, gm: (qk.forward(x, gm, 1e-6, cos, sin, interleaved)[0] * dy).sum()
    g = np.random.default_rng(4)
    for _ in range(6):
        v = g.normal(size=x.shape)
        d = (f(x + 1e-6 * v, gamma) - f(x - 1e-6 * v, gamma)) / 2e-6
        np.testing.assert_allclose((dx * v).sum(), d, rtol=1e-7, atol=1e-8)
    if norm:
        for i in range(gamma.size):
            v = np.eye(gamma.size)[i]
            np.testing.assert_allclose(dgamma[i], (f(x, gamma + 1e-6 * v) - f(x, gamma - 1e-6 * v)) / 2e-6, atol=1e-8)


def test_gradient_is_orthogonal_to_the_head_without_eps():
    # n does not change with the head's length, so neither does anything along it
    x, gamma, cos, sin, dy = _case(5)
    dx = qk.backward(dy, x, gamma, 0.0, cos, sin)[0]
    np.testing.assert_allclose((dx * x).sum(-1), 0.0, atol=1e-13)


def test_band_holds_a_binary32_evaluation():
    x, gamma, cos, sin, _ = _case(6, T=64, H=4, D=64, R=64)
    f = np.float32
    x = bf16.to_f32(bf16.from_f64_rne(x)).astype(np.float64)
    gamma = bf16.to_f32(bf16.from_f64_rne(gamma)).astype(np.float64)
    cos, sin = cos.astype(f).astype(np.float64), sin.astype(f).astype(np.float64)
    y, tol = qk.forward(x, gamma, 1e-6, cos, sin)
    r = f(1) / np.sqrt((x.astype(f) ** 2).sum(-1, keepdims=True, dtype=f) / f(64) + f(1e-6))
    n = x.astype(f) * r * gamma.astype(f)
    a, b = n[..., :32], n[..., 32:]
    c, s = cos[:, None].astype(f), sin[:, None].astype(f)
    got = np.concatenate((a * c - b * s, b * c + a * s), -1)
    assert (np.abs(got - y) <= tol).all()
    mid, lo, hi = (bf16.to_f32(v) for v in qk.band(y, tol))
    assert (lo <= mid).all() and (mid <= hi).all() and (lo == hi).mean() > 0.99
