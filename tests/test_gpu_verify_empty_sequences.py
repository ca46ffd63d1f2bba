"""Verification of drafted tokens over batches with sequences that have no rows
(an idle slot of a serving batch) ahead of others: they take no row of the draft's,
so that the other sequences' results are those of a batch without them."""

import numpy as np
import pytest

from oracle import verify as vf

from gpu_util import host, to_dev

pytestmark = pytest.mark.gpu

LG, PR = vf.LOGITS, vf.PROBS


@pytest.fixture(scope="module")
def P():
    from paper_2608_27370_amd import puro
    puro.lib()
    return puro


def soft(x):
    e = np.exp(x - x.max(-1, keepdims=True))
    return e / e.sum(-1, keepdims=True)


def batch(seed, rows, V, kind):
    """Targets, drafts near them, ids drawn from the drafts, random numbers; of the sequences that have rows."""
    g = np.random.default_rng(seed)
    full = np.array([n for n in rows if n])
    T = int(full.sum())
    last = np.zeros(T, bool)
    last[np.cumsum(full) - 1] = True
    z = g.normal(size=(T, V)) * 2
    zq = z[~last] + 0.5 * g.normal(size=(int((~last).sum()), V))
    ids = np.zeros(T, np.int32)
    ids[~last] = [g.choice(V, p=r) for r in soft(zq)]
    if kind == PR:
        z, zq = soft(z), soft(zq)
    return z.astype(np.float32), zq.astype(np.float32), ids, g.random(T).astype(np.float32), g.random(len(full)).astype(np.float32)


def offsets(rows):
    return np.concatenate([[0], np.cumsum(rows)]).astype(np.int32)


def run(P, z, zq, ids, off, u, us, kind):
    import torch
    tokens = torch.full((len(ids),), -9, dtype=torch.int32, device="cuda")
    tokens, accepted = P.verify_drafts(to_dev(z), None if zq is None else to_dev(zq), to_dev(ids), to_dev(off), to_dev(u), to_dev(us),
                                       kind=kind, tokens=tokens)
    return host(tokens).tolist(), host(accepted)


ROWS = [[0, 2], [3, 0, 3], [0, 0, 5, 0, 1, 4, 0], [1, 0, 1, 0, 2], [0] * 70 + [3, 0, 2], [2, 0] * 300 + [4], [0, 3, 0, 2, 1] * 400]


@pytest.mark.parametrize("kind", [LG, PR])
@pytest.mark.parametrize("rows", ROWS, ids=lambda r: "%d_sequences" % len(r))
def test_the_others_are_as_without_the_empty_ones(P, rows, kind):
    some = np.array(rows) > 0
    for drafted in (True, False):
        z, zq, ids, u, us = batch(len(rows), rows, 53, kind)
        zq = zq if drafted else None
        all_us = np.full(len(rows), 0.5, np.float32)
        all_us[some] = us
        got, kept = run(P, z, zq, ids, offsets(rows), u, all_us, kind)
        want, alone = run(P, z, zq, ids, offsets([n for n in rows if n]), u, us, kind)
        assert np.array_equal(kept[some], alone) and not kept[~some].any()
        assert np.array_equal(got, want)
        w = vf.verify(z.astype(np.float64), None if zq is None else zq.astype(np.float64), ids, offsets(rows), u, all_us, kind, 1.0,
                      np.full(len(ids), -9))
        assert np.array_equal(got, w[0]) and np.array_equal(kept, w[1])


@pytest.mark.parametrize("kind", [LG, PR])
def test_pieces_of_a_large_vocabulary(P, kind):
    rows = [0, 4, 0, 0, 3, 1, 0, 2]
    z, zq, ids, u, us = batch(3, rows, 20011, kind)
    all_us = np.full(len(rows), 0.5, np.float32)
    all_us[np.array(rows) > 0] = us
    got, kept = run(P, z, zq, ids, offsets(rows), u, all_us, kind)
    want, alone = run(P, z, zq, ids, offsets([n for n in rows if n]), u, us, kind)
    assert got == want and kept[np.array(rows) > 0].tolist() == alone.tolist()


@pytest.mark.parametrize("kind", [LG, PR])
def test_draft_rows_that_are_not_there(P, kind):
    """Fewer rows of the draft's than the sequences' drafts: those that have theirs are verified, the others refused."""
    rows = [0, 3, 0, 2]
    z, zq, ids, u, us = batch(8, rows, 40, kind)
    us = np.full(4, 0.5, np.float32)
    for n, want in ((3, [False, False]), (2, [False, True]), (1, [True, True])):
        kept = run(P, z, zq[:n], ids, offsets(rows), u, us, kind)[1]
        assert (kept[[1, 3]] == -1).tolist() == want and not kept[[0, 2]].any(), n


@pytest.mark.parametrize("kind", [LG, PR])
def test_a_graph_replayed_with_other_slots_idle(P, kind):
    import torch
    plans = [[2, 0, 3, 1], [0, 3, 0, 3], [3, 3, 0, 0], [1, 1, 1, 3]]
    T, V = 6, 300
    bufs = [torch.zeros(T, V, device="cuda"), torch.zeros(T, V, device="cuda"), torch.zeros(T, dtype=torch.int32, device="cuda"),
            to_dev(offsets(plans[0])), torch.zeros(T, device="cuda"), torch.full((4,), 0.5, device="cuda")]
    tokens, accepted = torch.zeros(T, dtype=torch.int32, device="cuda"), torch.zeros(4, dtype=torch.int32, device="cuda")

    def call():
        P.verify_drafts(*bufs, kind=kind, tokens=tokens, accepted=accepted)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        call()
    torch.cuda.current_stream().wait_stream(side)
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        call()
    for r, rows in enumerate(plans * 2):
        z, zq, ids, u, _ = batch(20 + r, rows, V, kind)
        bufs[0].copy_(to_dev(z))
        bufs[1][: len(zq)].copy_(to_dev(zq))
        for b, v in ((bufs[2], ids), (bufs[3], offsets(rows)), (bufs[4], u)):
            b.copy_(to_dev(v))
        tokens.fill_(-9)
        g.replay()
        torch.cuda.synchronize()
        want = vf.verify(z.astype(np.float64), zq.astype(np.float64), ids, offsets(rows), u, np.full(4, 0.5, np.float32), kind, 1.0,
                         np.full(T, -9))
        assert host(tokens).tolist() == want[0].tolist() and host(accepted).tolist() == want[1].tolist(), rows
    del g
