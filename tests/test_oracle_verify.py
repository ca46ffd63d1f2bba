"""Pins of the verification oracle (oracle/verify.py)."""

import numpy as np
import pytest
from scipy.special import softmax

from oracle import verify as vf


@pytest.mark.parametrize("kind", [vf.LOGITS, vf.PROBS])
def test_the_kept_or_drawn_token_is_distributed_as_the_target(kind):
    """One draft, its id drawn from q: over a grid of both random numbers the first token's frequencies are p."""
    g = np.random.default_rng(1)
    z, zq = g.normal(size=6) * 1.5, g.normal(size=6) * 1.5
    p, q = softmax(z / 0.7), softmax(zq / 0.7)
    rows, drafts = (np.stack([z, z]), zq[None]) if kind == vf.LOGITS else (np.stack([p, p]), q[None])
    grid = (np.arange(60) + 0.5) / 60
    found = np.zeros(6)
    for d in range(6):
        for u in grid:
            for us in grid:
                kept, token = vf.sequence(rows, drafts, np.array([d, -7]), np.array([u, 0.5]), us, kind, 0.7)
                found[d if kept else token] += q[d] / grid.size ** 2
    assert np.abs(found - p).max() < 2.0 / 60


def test_drafts_without_probabilities():
    """q = 1 at the id: kept with probability p(d), else drawn from the others."""
    p = np.array([0.1, 0.6, 0.0, 0.3])
    rows = np.stack([p, p])
    assert vf.sequence(rows, None, [1, 0], [0.59, 0], 0.95, vf.PROBS, 1.0) == (1, 3)
    for us, want in ((0.0, 0), (0.24, 0), (0.26, 3), (0.999, 3)):
        assert vf.sequence(rows, None, [1, 0], [0.61, 0], us, vf.PROBS, 1.0) == (0, want)
    assert vf.sequence(rows, None, [2, 0], [0.0, 0], 0.5, vf.PROBS, 1.0)[0] == 0          # p(d) = 0 is never kept


def test_equal_distributions_keep_everything_and_have_nothing_left():
    p = np.array([[0.25, 0.5, 0.25]] * 3)
    assert vf.sequence(p, p[:2], [0, 1, 9], [0.999, 0.999, 0], 0.8, vf.PROBS, 1.0) == (2, 2)
    # (u = 1 is outside the range that is asked for; nothing is left over then, so p is drawn from)
    assert vf.sequence(p, p[:2], [0, 1, 9], [1.0, 0, 0], 0.3, vf.PROBS, 1.0) == (0, 1)


def test_temperature_zero():
    z = np.array([[1.0, 3.0, 3.0], [5.0, 2.0, 1.0], [0.0, 0.0, 0.0]])
    assert vf.sequence(z, None, [1, 0, 5], None, None, vf.LOGITS, 0.0) == (2, 0)
    assert vf.sequence(z, None, [2, 0, 5], None, None, vf.LOGITS, 0.0) == (0, 1)
    z[0, 0] = np.nan
    assert vf.sequence(z, None, [1, 0, 5], None, None, vf.LOGITS, 0.0) == (0, -1)


def test_rows_without_probability_and_invalid_offsets():
    z = np.array([[0.0, 1.0], [-np.inf, -np.inf], [0.0, 0.0], [np.inf, 0.0]])
    out, acc = vf.verify(z, None, np.array([1, 1, 0, 0]), [0, 2, 2, 1, 9], np.zeros(4), np.full(4, 0.9), vf.LOGITS, 1.0,
                         np.full(4, 77))
    assert list(acc) == [1, 0, -1, -1] and list(out) == [1, -1, 77, 77]
    assert vf.sequence(z[3:], None, [0], [0.0], 0.1, vf.LOGITS, 1.0) == (0, -1)
