"""Pins of the distillation oracle (oracle/lm_distill.py)."""

import numpy as np
import pytest
from scipy.special import rel_entr, softmax

from oracle import bf16, lm_distill as ld
from oracle.lm_head import logits


def _case(seed, M=5, V=40, K=16, k=6):
    g = np.random.default_rng(seed)
    X, W = bf16.from_f64_rne(g.normal(size=(M, K))), bf16.from_f64_rne(g.normal(size=(V, K)) * 0.4)
    ids = np.argsort(g.random((M, V)), axis=1)[:, :k]
    return X, W, ids, g.normal(size=(M, k)) * 2, g


@pytest.mark.parametrize("tau", [1.0, 0.5, 3.0])
def test_relative_entropy_of_all_entries(tau):
    # a teacher known in full: the divergence of two distributions over the vocabulary
    X, W, _, _, g = _case(1)
    ids = np.tile(np.arange(40), (5, 1))
    t = g.normal(size=(5, 40))
    z, _ = logits(X, W)
    want = rel_entr(softmax(t / tau, 1), softmax(z / tau, 1)).sum(1)
    np.testing.assert_allclose(ld.forward(X, W, ids, t, tau, ld.LOGITS)["loss"], want, rtol=1e-12)
    np.testing.assert_allclose(ld.forward(X, W, ids, softmax(t / tau, 1), tau, ld.PROBS)["loss"], want, rtol=1e-12)


def test_one_entry_is_the_cross_entropy():
    X, W, ids, t, _ = _case(2, k=1)
    z, _ = logits(X, W)
    ce = np.log(np.exp(z).sum(1)) - np.take_along_axis(z, ids, 1)[:, 0]
    np.testing.assert_allclose(ld.forward(X, W, ids, t, 1.0, ld.LOGITS)["loss"], ce, rtol=1e-12)
    dz = ld.gradient(X, W, ids, t, 1.0, ld.LOGITS, np.ones(5))
    onehot = np.eye(40)[ids[:, 0]]
    np.testing.assert_allclose(dz, softmax(z, 1) - onehot, atol=1e-14)


def test_a_teacher_like_the_student_costs_nothing():
    X, W, _, _, _ = _case(3)
    z, _ = logits(X, W)
    ids = np.tile(np.arange(40), (5, 1))
    np.testing.assert_allclose(ld.forward(X, W, ids, z, 2.0, ld.LOGITS)["loss"], 0.0, atol=1e-14)
    np.testing.assert_allclose(ld.gradient(X, W, ids, z, 2.0, ld.LOGITS, np.ones(5)), 0.0, atol=1e-15)


def test_entries_that_do_not_count():
    X, W, ids, t, _ = _case(4)
    more = np.concatenate((ids, [[-1, 40, 2 ** 31 - 1]] * 5), 1)
    tt = np.concatenate((t, np.full((5, 3), 99.0)), 1)
    a, b = ld.forward(X, W, ids, t, 1.5, ld.LOGITS), ld.forward(X, W, more, tt, 1.5, ld.LOGITS)
    np.testing.assert_allclose(a["loss"], b["loss"], rtol=1e-14)
    assert (b["z_top"][:, 6:] == 0).all()
    none = np.full_like(ids, -1)
    for kind in (ld.LOGITS, ld.PROBS):
        assert (ld.forward(X, W, none, t, 1.0, kind)["loss"] == 0).all()
        assert (ld.gradient(X, W, none, t, 1.0, kind, np.ones(5)) == 0).all()
    assert (ld.forward(X, W, ids, np.full_like(t, -np.inf), 1.0, ld.LOGITS)["loss"] == 0).all()
    # all at the lowest value: as good as any other constant
    low = ld.forward(X, W, ids, np.full_like(t, np.finfo(np.float32).min), 0.5, ld.LOGITS)["loss"]
    np.testing.assert_allclose(low, ld.forward(X, W, ids, np.zeros_like(t), 0.5, ld.LOGITS)["loss"], rtol=1e-14)


@pytest.mark.parametrize("kind", [ld.LOGITS, ld.PROBS])
@pytest.mark.parametrize("tau", [1.0, 2.5])
def test_gradient_by_differences(kind, tau):
    """Along X and W through dX = dz W and dW = dz^T X, with an id given twice and weights that do not add up to 1."""
    X, W, ids, t, g = _case(5)
    ids[:, 1] = ids[:, 0]
    if kind == ld.PROBS:
        t = softmax(t, 1) * 0.8
    dloss = g.normal(size=5)
    dz = ld.gradient(X, W, ids, t, tau, kind, dloss, 0.5)
    x, w = (bf16.to_f32(v).astype(np.float64) for v in (X, W))

    def f(x, w):
        a = x @ w.T / tau
        q, log_q, _ = ld.teacher(ids, t, 40, tau, kind)
        lse = np.log(np.exp(a).sum(1, keepdims=True))
        return 0.5 * (dloss * (q * (log_q - np.take_along_axis(a, ids, 1) + lse)).sum(1)).sum()
    for _ in range(5):
        u, v = g.normal(size=x.shape), g.normal(size=w.shape)
        d = (f(x + 1e-6 * u, w) - f(x - 1e-6 * u, w)) / 2e-6
        np.testing.assert_allclose(((dz @ w) * u).sum(), d, rtol=1e-6, atol=1e-8)
        d = (f(x, w + 1e-6 * v) - f(x, w - 1e-6 * v)) / 2e-6
        np.testing.assert_allclose(((dz.T @ x) * v).sum(), d, rtol=1e-6, atol=1e-8)


def test_band_holds_the_value():
    X, W, ids, t, _ = _case(6)
    f = ld.forward(X, W, ids, t, 2.0, ld.LOGITS)
    mid, lo, hi = (bf16.to_f32(v) for v in ld.dz_band(f, 2.0, np.ones(5), 1.0))
    dz = ld.gradient(X, W, ids, t, 2.0, ld.LOGITS, np.ones(5))
    assert (lo <= mid).all() and (mid <= hi).all()
    assert (np.abs(mid - dz) <= 2.0 ** -8 * np.abs(dz)).all()
