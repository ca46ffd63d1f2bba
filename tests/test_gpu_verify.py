"""GPU parity of the verification of drafted tokens (puro_verify_drafts) against
the oracle (oracle/verify.py): tokens and counts equal. Both sum in binary64, with
exponentials to 4.4e-11 here; an entry of the running sum would have to lie within
about 10^-10 of the random number's share for the two to choose differently."""

import numpy as np
import pytest

from oracle import bf16, verify as vf

from gpu_util import host, to_dev

pytestmark = pytest.mark.gpu

LG, PR = vf.LOGITS, vf.PROBS


@pytest.fixture(scope="module")
def P():
    from paper_2608_27370_amd import puro
    puro.lib()
    return puro


class Batch:
    """Sequences with the given numbers of rows; the draft's logits near the target's, ids drawn from the draft's."""

    def __init__(self, seed, rows, V, kind, dtype, tau, drafted=True, spare=0):
        g = np.random.default_rng(seed)
        self.kind, self.dtype, self.tau, self.V = kind, dtype, tau, V
        T, B = sum(rows), len(rows)
        self.offsets = np.concatenate([[0], np.cumsum(rows)]).astype(np.int32)
        z = g.normal(size=(T + spare, V)) * 2 - np.log1p(g.permutation(V))
        z[:, g.random(V) < 0.1] = -np.inf
        z[:, 0] = 0.0
        last = np.zeros(T + spare, bool)
        last[self.offsets[1:][np.array(rows) > 0] - 1] = True
        last[T:] = True
        zq = z[~last] + 0.7 * g.normal(size=(int((~last).sum()), V))
        t = tau if tau else 1.0
        soft = lambda x: np.exp((x - x.max(-1, keepdims=True)) / t) / np.exp((x - x.max(-1, keepdims=True)) / t).sum(-1, keepdims=True)  # noqa: E731
        self.ids = np.full(T + spare, 2 ** 31 - 1, np.int64)
        self.ids[~last] = [g.choice(V, p=r) for r in soft(zq)]
        if tau == 0:
            best = z[~last].argmax(1)
            self.ids[~last] = np.where(g.random(best.size) < 0.7, best, self.ids[~last])
        self.ids = self.ids.astype(np.int32)
        if kind == PR:
            z, zq = soft(z), soft(zq)
        self.target, self.draft = self.store(z), self.store(zq) if drafted else None
        self.u, self.us = g.random(T + spare).astype(np.float32), g.random(B).astype(np.float32)

    def store(self, x):
        """As the type holds it (BF16: bit patterns)."""
        return x.astype(np.float32) if self.dtype == "fp32" else bf16.from_f64_rne(x)

    def values(self, x):
        return None if x is None else x.astype(np.float64) if self.dtype == "fp32" else bf16.to_f32(x).astype(np.float64)

    def up(self, x, pitch=None, shift=0):
        """On the device, with a row pitch and a first element that `shift` elements from an aligned address precede."""
        import torch
        if x is None:
            return None
        pitch = self.V if pitch is None else pitch
        room = np.full(shift + x.shape[0] * pitch, 0x7FC0 if self.dtype == "bf16" else np.nan, x.dtype)
        room[shift:].reshape(x.shape[0], pitch)[:, :self.V] = x
        d = to_dev(room.view(np.int16)).view(torch.bfloat16) if self.dtype == "bf16" else to_dev(room)
        return d[shift:].view(x.shape[0], pitch)[:, :self.V]

    def want(self, before=-9):
        return vf.verify(self.values(self.target), self.values(self.draft), self.ids, self.offsets, self.u, self.us, self.kind,
                         self.tau, np.full(len(self.ids), before))

    def run(self, P, pitch=None, shift=0, before=-9):
        import torch
        tokens = torch.full((len(self.ids),), before, dtype=torch.int32, device="cuda")
        return P.verify_drafts(self.up(self.target, pitch, shift), self.up(self.draft, pitch, shift), to_dev(self.ids),
                               to_dev(self.offsets), to_dev(self.u), to_dev(self.us), temperature=self.tau, kind=self.kind,
                               tokens=tokens)

    def check(self, P, **kw):
        tokens, accepted = self.run(P, **kw)
        want = self.want()
        assert host(accepted).tolist() == want[1].tolist()
        assert host(tokens).tolist() == want[0].tolist()
        return want


ROWS = [[1], [2], [5], [1, 4, 2, 8, 3, 1], [9] * 7]
VOCABULARIES = [1, 2, 7, 255, 1000, 8191, 8192, 8193, 20011]


@pytest.mark.parametrize("V", VOCABULARIES)
@pytest.mark.parametrize("kind", [LG, PR])
@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
def test_batches(P, V, kind, dtype):
    for i, rows in enumerate(ROWS):
        for drafted in (True, False):
            Batch(V + i, rows, V, kind, dtype, (1.0, 0.6, 2.5)[i % 3], drafted).check(P)


def test_drafts_are_kept_and_refused(P):
    """(that the batches above reach both ends)"""
    kept = np.concatenate([Batch(s, [6] * 30, 500, LG, "fp32", 1.0).check(P)[1] for s in range(3)])
    assert set(kept.tolist()) == set(range(6))


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("V,pitch,shift", [(1000, 1003, 0), (1001, 1001, 1), (8195, 8201, 3), (8200, 8208, 5)])
def test_pitches_and_unaligned_rows(P, dtype, V, pitch, shift):
    for kind in (LG, PR):
        Batch(V, [3, 1, 4], V, kind, dtype, 0.9).check(P, pitch=pitch, shift=shift)
    Batch(V, [3, 1, 4], V, LG, dtype, 0.0).check(P, pitch=pitch, shift=shift)


@pytest.mark.parametrize("V", VOCABULARIES)
@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
def test_temperature_zero(P, V, dtype):
    b = Batch(V, [4, 1, 7, 2], V, LG, dtype, 0.0)
    want = b.check(P)
    # random numbers and the draft's rows are not needed then
    import torch
    tokens = torch.full((len(b.ids),), -9, dtype=torch.int32, device="cuda")
    tokens, accepted = P.verify_drafts(b.up(b.target), None, to_dev(b.ids), to_dev(b.offsets), temperature=0.0, tokens=tokens)
    assert host(tokens).tolist() == want[0].tolist() and host(accepted).tolist() == want[1].tolist()


@pytest.mark.parametrize("kind,dtype,tau", [(LG, "bf16", 0.8), (LG, "fp32", 1.0), (PR, "fp32", 1.0), (LG, "bf16", 0.0)])
def test_many_rows_of_a_large_vocabulary(P, kind, dtype, tau):
    """(where the rows' pieces are the longer ones)"""
    Batch(21, [1, 6, 3, 5] * 8, 150001, kind, dtype, tau).check(P)


@pytest.mark.parametrize("tau", [2.0 ** -20, 1e-3, 0.05, 300.0, 2.0 ** 20])
def test_extreme_temperatures(P, tau):
    for drafted in (True, False):
        Batch(31, [5, 1, 3, 4], 9001, LG, "fp32", tau, drafted).check(P)


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("shift", [3000.0, -9000.0, 1e5, -3e7, 1e30, -3.3e38])
def test_logits_far_from_zero(P, dtype, shift):
    """Rows moved by a large amount (as the type holds them then), some of their entries as large the other way."""
    b = Batch(32, [4, 2, 6], 5000, LG, dtype, 0.9)
    for name in ("target", "draft"):
        v = b.values(getattr(b, name))
        v = np.where(np.isfinite(v), v * (1 + abs(shift) * 2.0 ** -9) + shift, v)
        v[:, 7] = -abs(shift)
        setattr(b, name, b.store(np.clip(v, -3.38e38, 3.38e38) if shift < 0 or shift > 1e30 else v))
    b.u[:] = np.linspace(0, 0.9, b.u.size)
    b.check(P)


def test_ties_go_to_the_lowest_id(P):
    b = Batch(1, [3, 2], 20000, LG, "bf16", 0.0)
    b.target[:] = 0
    b.target[:, 9000] = b.target[:, 17] = b.target[:, 12000] = 0x4000
    b.ids[:] = 17
    assert b.check(P)[1].tolist() == [2, 1]
    b.ids[:] = 9000
    assert b.check(P)[1].tolist() == [0, 0]


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
def test_the_smallest_values_and_signed_zeros(P, dtype):
    b = Batch(35, [1] * 6, 3001, LG, dtype, 0.0)
    b.draft = None
    word = np.uint16 if dtype == "bf16" else np.uint32
    x = np.full(b.target.shape, 0xFF80 if dtype == "bf16" else 0xFF800000, word)
    sign = 0x8000 if dtype == "bf16" else 0x80000000
    x[0, [7, 2999]] = 1, 2                           # the two smallest positive numbers
    x[1, [7, 2999]] = sign | 2, sign | 1
    x[2, [1030, 2]] = 0, sign                        # zeros are equal: the first of them
    x[3, [1030, 2]] = sign, 0
    x[4, 3000] = sign
    x[5] = sign | 3
    b.target = x.view(b.target.dtype)
    assert host(b.run(P)[0]).tolist() == b.want()[0].tolist() == [2999, 2999, 2, 2, 3000, 0]


def test_many_drafts_of_one_sequence(P):
    b = Batch(3, [200, 1, 70], 300, LG, "fp32", 1.0)
    b.check(P)
    b.u[:] = 0.0                                     # every draft that has a probability is kept
    assert b.check(P)[1].tolist() == [199, 0, 69]


@pytest.mark.parametrize("kind", [LG, PR])
def test_random_numbers_at_their_ends(P, kind):
    for u in (0.0, np.float32(1 - 2.0 ** -24), 1.0):
        for us in (0.0, np.float32(1 - 2.0 ** -24), 1.0):
            b = Batch(5, [3, 1, 2, 4], 9001, kind, "fp32", 1.0)
            b.u[:], b.us[:] = u, us
            b.check(P)


def test_draft_like_the_target(P):
    """p = q: everything is kept, and where a draft is refused all the same nothing is left over: p is drawn from."""
    b = Batch(6, [4, 4, 2], 3000, PR, "fp32", 1.0)
    b.draft = b.target[[0, 1, 2, 4, 5, 6, 8]].copy()
    assert b.check(P)[1].tolist() == [3, 3, 1]
    b.u[:] = 1.0
    assert b.check(P)[1].tolist() == [0, 0, 0]


@pytest.mark.parametrize("low", [-np.inf, -1e30, -5000.0])
@pytest.mark.parametrize("drafted", [True, False])
def test_nothing_left_over_behind_masked_entries(P, low, drafted):
    """Nothing is left over and the first thousands of entries have no probability: the least random number takes the first that has (without
    the draft's predictions everything is left over of an id that is none)."""
    b = Batch(33, [2, 3], 7000, LG, "fp32", 1.0)
    b.target[:, :5000] = low
    b.target[:, 5000] = 0.0
    b.draft = b.target[[0, 2, 3]].copy() if drafted else None
    b.ids[:] = b.V
    for us in (0.0, 1e-30, 0.5):
        b.us[:] = us
        tokens, accepted = b.check(P)
        assert accepted.tolist() == [0, 0] and tokens[[0, 2]].min() >= 5000


@pytest.mark.parametrize("tau", [1.0, 0.0])
@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
def test_special_logits(P, tau, dtype):
    b = Batch(7, [3, 3, 3, 3, 3, 3], 9000, LG, dtype, tau)
    bad = np.array([0x7FC0, 0x7F80, 0xFF80], np.uint16)
    nan, inf, ninf = bad if dtype == "bf16" else bf16.to_f32(bad)
    b.u[:] = 0.0
    b.target[0, 8999] = nan                          # a NaN in the row of the first draft
    b.target[4, 3] = inf                             # an infinity in the second's
    b.target[6] = ninf                               # nothing but -infinity
    b.target[11] = ninf                              # the same in a last row
    b.target[12] = ninf                              # one token left, which is not the draft
    b.target[12, (int(b.ids[12]) + 1) % 9000] = 0
    b.ids[15] = 9000                                 # ids outside the vocabulary
    b.ids[16] = -1
    b.check(P)
    if tau:
        b.draft[0, 5] = nan
        b.draft[3, :] = ninf
        b.check(P)


def test_special_probabilities(P):
    b = Batch(8, [2, 2, 2, 1, 1, 1], 8500, PR, "fp32", 1.0)
    b.u[:] = 0.999
    b.target[0, 8400] = np.nan
    b.draft[1, 20] = np.nan
    b.draft[2, 30] = np.inf
    b.target[6] = 0.0
    b.target[7, 2] = np.inf
    b.target[8] = 0.0
    b.target[8, 8499] = 1e-30                        # one entry, the last
    b.check(P)


def test_sequences_without_rows_and_rows_behind_the_last(P):
    for kind in (LG, PR):
        b = Batch(9, [3, 2, 4, 0, 0], 1200, kind, "fp32", 1.0, spare=6)
        tokens = b.check(P)[0]
        assert (tokens[9:] == -9).all()
    Batch(9, [3, 2, 0], 1200, LG, "bf16", 0.0, spare=3).check(P)
    b = Batch(10, [0, 0], 50, LG, "fp32", 1.0, spare=4)
    assert b.check(P)[1].tolist() == [0, 0]


@pytest.mark.parametrize("tau", [1.0, 0.0])
def test_invalid_offsets(P, tau):
    b = Batch(11, [3, 2, 4, 1], 600, LG, "fp32", tau)
    for off in ([0, 3, 2, 9, 10], [-1, 3, 5, 9, 10], [0, 3, 5, 11, 10], [2 ** 31 - 1, -2 ** 31, 5, 9, 10], [0, 3, 3, 9, 10],
                [0, 0, 0, 9, 10], [0, 10, 10, 10, 10]):
        b.offsets = np.array(off, np.int32)
        if tau == 0:
            b.draft = None
        b.check(P)


@pytest.mark.parametrize("tau", [1.0, 0.0])
@pytest.mark.parametrize("B", [512, 513, 1100, 3001])
def test_many_sequences_some_of_them_invalid(P, B, tau):
    g = np.random.default_rng(B)
    b = Batch(34, g.integers(0, 4, B).tolist(), 41, LG, "fp32", tau, drafted=tau != 0)
    if tau == 0:
        b.draft = None
    b.check(P)
    for k in g.integers(1, B, 6):                    # jumps ahead: the sequences behind begin before them
        b.offsets[k] += int(g.integers(1, 12))
        b.check(P)
    b.offsets[B // 2] = -1
    b.check(P)
    b.offsets[3] = 2 ** 31 - 1
    assert (b.check(P)[1][4:] == -1).all()


@pytest.mark.parametrize("kind,tau,drafted", [(LG, 0.0, False), (LG, 1.0, True), (LG, 1.0, False), (PR, 1.0, True)])
def test_tokens_over_the_ids(P, kind, tau, drafted):
    b = Batch(36, [70, 1, 9, 300, 5], 50, kind, "fp32", tau, drafted)
    if tau == 0:
        b.ids[:300] = np.where(np.arange(300) < 200, b.values(b.target)[:300].argmax(1), b.ids[:300])
    want, ids = b.want(), to_dev(b.ids)
    for _ in range(5):
        ids.copy_(to_dev(b.ids))
        tokens, accepted = P.verify_drafts(b.up(b.target), b.up(b.draft), ids, to_dev(b.offsets), to_dev(b.u), to_dev(b.us),
                                           temperature=tau, kind=kind, tokens=ids)
        assert tokens is ids and host(ids).tolist() == want[0].tolist() and host(accepted).tolist() == want[1].tolist()


def test_no_sequences_and_no_drafts_at_all(P):
    import torch
    z = torch.zeros(0, 40, device="cuda")
    i, f = torch.zeros(0, dtype=torch.int32, device="cuda"), torch.zeros(0, device="cuda")
    tokens, accepted = P.verify_drafts(z, None, i, torch.zeros(1, dtype=torch.int32, device="cuda"), f, f)
    assert tokens.shape == (0,) and accepted.shape == (0,)
    tokens, accepted = P.verify_drafts(z, z, i, torch.zeros(3, dtype=torch.int32, device="cuda"), f, torch.zeros(2, device="cuda"))
    assert accepted.tolist() == [0, 0]
    b = Batch(12, [1, 1, 1], 40, LG, "fp32", 1.0)
    assert b.draft.shape == (0, 40)
    b.check(P)
    # (a draft tensor without rows has none for a sequence of two)
    b.offsets = np.array([0, 2, 3, 3], np.int32)
    assert b.check(P)[1].tolist() == [-1, 0, 0]


def test_refusals_of_the_binding(P):
    import torch
    b = Batch(13, [2, 1], 40, LG, "fp32", 1.0)
    a = [b.up(b.target), b.up(b.draft), to_dev(b.ids), to_dev(b.offsets), to_dev(b.u), to_dev(b.us)]
    for i, t in ((0, a[0].double()), (1, a[1].bfloat16()), (1, a[1][:, :39]), (2, a[2].long()), (2, a[2][:2]), (3, a[3].float()),
                 (4, a[4][:2]), (5, a[5][:1]), (0, a[0].cpu())):
        with pytest.raises((TypeError, ValueError)):
            P.verify_drafts(*a[:i], t, *a[i + 1:])
    for kw in (dict(tokens=torch.zeros(2, dtype=torch.int32, device="cuda")), dict(accepted=torch.zeros(2, device="cuda"))):
        with pytest.raises((TypeError, ValueError)):
            P.verify_drafts(*a, **kw)
    for kw in (dict(temperature=-1.0), dict(kind=2)):
        with pytest.raises(P.PuroError):
            P.verify_drafts(*a, **kw)
    with pytest.raises(P.PuroError):
        P.verify_drafts(*a[:4])                      # random numbers are needed at this temperature


def test_two_graphs_and_a_side_stream(P):
    """Two captured batches, replayed in turn on other inputs with eager work between; each replay is the oracle's."""
    import torch
    made = []
    for seed, rows, V, tau in ((1, [3, 1, 5], 9000, 0.8), (2, [2, 2], 700, 1.0)):
        b = Batch(seed, rows, V, LG, "fp32", tau)
        bufs = [b.up(b.target), b.up(b.draft), to_dev(b.ids), to_dev(b.offsets), to_dev(b.u), to_dev(b.us)]
        tokens = torch.full((len(b.ids),), -9, dtype=torch.int32, device="cuda")
        accepted = torch.zeros(len(rows), dtype=torch.int32, device="cuda")
        call = lambda bufs=bufs, tau=tau, t=tokens, a=accepted: P.verify_drafts(*bufs, temperature=tau, tokens=t, accepted=a)  # noqa: E731
        side = torch.cuda.Stream()
        side.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(side):
            call()
        torch.cuda.current_stream().wait_stream(side)
        torch.cuda.synchronize()
        want = b.want()
        assert host(tokens).tolist() == want[0].tolist()
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            call()
        made.append((seed, rows, V, tau, bufs, tokens, accepted, g))
    for r in range(3):
        wants = []
        for seed, rows, V, tau, bufs, tokens, accepted, g in made:
            b = Batch(seed + 10 * (r + 1), rows, V, LG, "fp32", tau)
            for d, s in zip(bufs, (b.up(b.target), b.up(b.draft), to_dev(b.ids), to_dev(b.offsets), to_dev(b.u), to_dev(b.us))):
                d.copy_(s)
            tokens.fill_(-9)
            wants.append(b.want())
        for m in made:
            m[-1].replay()
        torch.cuda.synchronize()
        for m, w in zip(made, wants):
            assert host(m[5]).tolist() == w[0].tolist() and host(m[6]).tolist() == w[1].tolist()
        Batch(99 + r, [2, 3], 300, PR, "bf16", 1.0).check(P)
    del made


def test_int8_head_then_verification(P):
    """The LM head in int8 over a batch's drafted tokens, its logits straight into the verification."""
    import torch
    from oracle import int8
    K, V, rows = 64, 3001, [4, 2, 1]
    g = np.random.default_rng(3)
    W = P.quantize_int8(to_dev(bf16.from_f64_rne(g.normal(size=(V, K)) * 0.3).view(np.int16)).view(torch.bfloat16))
    X = to_dev(bf16.from_f64_rne(g.normal(size=(7, K))).view(np.int16)).view(torch.bfloat16)
    gamma = torch.ones(K, dtype=torch.bfloat16, device="cuda")
    h = P.rmsnorm_quantize_int8(X, gamma, 1e-6)
    z = P.int8_gemm(h["q"], h["scale"], W["q"], W["scale"], P.OUT_FP32)          # [7, V], rows padded to 3004
    ref, tol = int8.gemm(host(h["q"]), host(h["scale"]), host(W["q"]), host(W["scale"]))
    assert (np.abs(host(z) - ref) <= tol + 2.0 ** -24 * np.abs(ref)).all()
    b = Batch(4, rows, V, LG, "fp32", 1.0)
    b.target = host(z).astype(np.float32)
    b.draft = b.target[[0, 1, 2, 4]] + g.normal(size=(4, V)).astype(np.float32) * 0.5
    b.ids[[0, 1, 2, 4]] = b.draft.argmax(1)
    tokens = torch.full((7,), -9, dtype=torch.int32, device="cuda")
    tokens, accepted = P.verify_drafts(z, b.up(b.draft), to_dev(b.ids), to_dev(b.offsets), to_dev(b.u), to_dev(b.us), tokens=tokens)
    want = b.want()
    assert host(tokens).tolist() == want[0].tolist() and host(accepted).tolist() == want[1].tolist()
