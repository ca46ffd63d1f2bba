"""Pins of the verification oracle (oracle/verify.py) over batches with sequences
that have no rows: the draft's rows lie one after another, those of a sequence
without rows are none."""

import numpy as np
import pytest
from scipy.special import softmax

from oracle import verify as vf

V, TAU = 5, 0.7


@pytest.mark.parametrize("kind", [vf.LOGITS, vf.PROBS])
@pytest.mark.parametrize("rows,at", [([0, 2], 1), ([3, 0, 2], 2), ([0, 1, 0, 2, 0], 3)])
def test_behind_empty_sequences_the_token_is_distributed_as_the_target(kind, rows, at):
    """One draft of sequence `at`, its id drawn from its own q: over a grid of both random numbers its first token's
    frequencies are its p, whatever the rows of the sequences before hold."""
    g = np.random.default_rng(len(rows))
    T, B = sum(rows), len(rows)
    offsets = np.concatenate([[0], np.cumsum(rows)])
    drafts = sum(max(0, n - 1) for n in rows)
    z, zq = g.normal(size=(T, V)) * 1.5, g.normal(size=(drafts, V)) * 1.5
    t = int(offsets[at])
    mine = sum(max(0, n - 1) for n in rows[:at])                # its draft's row, counted
    p, q = softmax(z[t] / TAU), softmax(zq[mine] / TAU)
    target, draft = (z, zq) if kind == vf.LOGITS else (softmax(z / TAU, axis=1), softmax(zq / TAU, axis=1))
    grid = (np.arange(40) + 0.5) / 40
    found = np.zeros(V)
    ids, u, us = np.zeros(T, int), np.full(T, 0.5), np.full(B, 0.5)
    for d in range(V):
        ids[t] = d
        for u[t] in grid:
            for us[at] in grid:
                tokens, accepted = vf.verify(target, draft, ids, offsets, u, us, kind, TAU, np.full(T, -9))
                assert accepted[at] >= 0
                found[tokens[t]] += q[d] / grid.size ** 2
    assert np.abs(found - p).max() < 2.0 / 40


def test_the_others_are_as_without_the_empty_ones():
    g = np.random.default_rng(4)
    rows = [0, 3, 0, 0, 1, 4, 0, 2]
    full = [n for n in rows if n]
    T = sum(rows)
    z, zq = g.normal(size=(T, 30)) * 2, g.normal(size=(T - len(full), 30)) * 2
    ids, u = g.integers(0, 30, T), g.random(T) * 0.3
    us = g.random(len(rows))
    off = lambda r: np.concatenate([[0], np.cumsum(r)])          # noqa: E731
    a, na = vf.verify(z, zq, ids, off(rows), u, us, vf.LOGITS, 1.0, np.full(T, -9))
    b, nb = vf.verify(z, zq, ids, off(full), u, us[np.array(rows) > 0], vf.LOGITS, 1.0, np.full(T, -9))
    assert a.tolist() == b.tolist() and na[np.array(rows) > 0].tolist() == nb.tolist()
    assert not na[np.array(rows) == 0].any()


def test_draft_rows_that_are_not_there():
    z = np.zeros((3, 4))
    ids, u, us = np.zeros(3, int), np.zeros(3), np.zeros(3)
    tokens = np.full(3, -9)
    assert vf.verify(z, z[:1], ids, [0, 0, 1, 3], u, us, vf.LOGITS, 1.0, tokens)[1].tolist() == [0, 0, 1]
    assert vf.verify(z, z[:0], ids, [0, 0, 1, 3], u, us, vf.LOGITS, 1.0, tokens)[1].tolist() == [0, 0, -1]
