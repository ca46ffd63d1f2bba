"""Verification of drafted tokens against a target's probabilities, in float64.

Test infrastructure only (see the package docstring). The usual speculative
sampling rule: draft i of a sequence is kept while u q(d) < p(d); the first that
is not (or the place after all of them) takes the least v whose running sum of
max(p - q, 0) (of p after all of them, and where that is 0 everywhere) exceeds
u' times the whole, the last v with a share where rounding leaves none.
temperature 0: the largest logit, the lowest id among equals.

Parity unpinned by the paper (it drafts nothing); tests/test_oracle_verify.py
pins it by the distribution that it leaves, the target's own.
"""

import numpy as np

LOGITS, PROBS = 0, 1


def probabilities(row, kind, tau):
    row = np.asarray(row, dtype=np.float64)
    if kind == PROBS:
        return row
    with np.errstate(invalid="ignore", divide="ignore"):
        e = np.exp((row - row.max()) / tau)
        return e / e.sum()


def draw(rest, u):
    total = rest.sum()
    if not (total > 0 and np.isfinite(total)):
        return -1
    cum = np.cumsum(rest)
    hit = np.nonzero(cum > np.float64(u) * cum[-1])[0]
    return int(hit[0]) if len(hit) else int(np.nonzero(rest > 0)[0][-1])


def sequence(target, draft, ids, u, us, kind, tau):
    """(kept, token) of one sequence: target [n, V], draft [n - 1, V] or None, ids and u [n]."""
    n, V = target.shape
    if kind == LOGITS and tau == 0:
        best = [-1 if np.isnan(r).any() or r.max() in (np.inf, -np.inf) else int(r.argmax()) for r in target]
        kept = 0
        while kept < n - 1 and best[kept] >= 0 and best[kept] == ids[kept]:
            kept += 1
        return kept, best[kept]
    for i in range(n):
        p = probabilities(target[i], kind, tau)
        if i == n - 1:
            return i, draw(p, us)
        q = np.zeros(V)
        if draft is not None:
            q = probabilities(draft[i], kind, tau)
        elif 0 <= ids[i] < V:
            q[ids[i]] = 1.0
        if 0 <= ids[i] < V and np.float64(u[i]) * q[ids[i]] < p[ids[i]]:
            continue
        if not np.isfinite(p.sum()) or np.isnan(q).any():
            return i, -1
        with np.errstate(invalid="ignore"):
            rest = np.maximum(p - q, 0.0)
        return i, draw(rest if rest.sum() > 0 else p, us)


def verify(target, draft, ids, offsets, u, us, kind, tau, tokens):
    """(tokens, accepted); `tokens` holds what the rows behind the last sequence have. The draft's rows lie one after
    another like the target's, but for the last one of every sequence that has rows."""
    tokens, B, T = np.array(tokens), len(offsets) - 1, len(ids)
    accepted = np.zeros(B, np.int32)
    left_out = 0                     # last rows of the sequences before, which the draft has none for
    for b in range(B):
        lo, hi = int(offsets[b]), int(offsets[b + 1])
        first = lo - left_out
        left_out += lo != hi
        if lo < 0 or hi < lo or hi > T or max(offsets[:b + 1]) > lo or (draft is not None and hi - lo > 1 and (first < 0 or first + hi - lo - 1 > len(draft))):
            accepted[b] = -1
            continue
        if lo == hi:
            continue
        d = None if draft is None else draft[first:first + hi - lo - 1]
        kept, token = sequence(target[lo:hi], d, ids[lo:hi], u[lo:hi], us[b], kind, tau)
        accepted[b] = kept
        tokens[lo:hi] = -1
        tokens[lo:lo + kept] = ids[lo:lo + kept]
        tokens[lo + kept] = token
    return tokens, accepted
