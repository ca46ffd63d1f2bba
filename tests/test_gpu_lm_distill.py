"""GPU parity of the LM head's distillation loss (puro_lm_head_distill_fwd,
puro_lm_head_distill_bwd) against the oracle (oracle/lm_distill.py): lse, loss
and z_top within its allowances, dX and dW within the GEMMs' 1e-5 sum |ab| plus
what the BF16 values that the oracle accepts for dz can move them."""

import numpy as np
import pytest

from oracle import bf16, lm_distill as ld

from gpu_util import bf16_bits, check_bf16, check_fp32, host, to_dev, to_dev_bf16

pytestmark = pytest.mark.gpu

L, PR = ld.LOGITS, ld.PROBS


@pytest.fixture(scope="module")
def P():
    from paper_2608_27370_amd import puro
    puro.lib()
    return puro


def f64(b):
    return bf16.to_f32(np.asarray(b, dtype=np.uint16)).astype(np.float64)


class Case:
    """Inputs with what is awkward among them: entries that do not count (-1, V, the largest and smallest int32),
    an id given twice, a row without entries, a row of teacher logits -infinity, one at the lowest value."""

    def __init__(self, seed, M, V, K, k, kind=L, plain=False):
        g = np.random.default_rng(seed)
        self.M, self.V, self.K, self.k, self.kind = M, V, K, k, kind
        self.X = bf16.from_f64_rne(g.standard_t(3, (M, K)))
        self.W = bf16.from_f64_rne(g.normal(size=(V, K)) * min(0.3, 1.0 / np.sqrt(K)))
        self.ids = (g.random((M, k)) ** 3 * V).astype(np.int64)
        self.t = g.normal(size=(M, k)) * 3
        if not plain:
            if k > 2:
                self.ids[:, 1] = np.where(g.random(M) < 0.5, self.ids[:, 0], self.ids[:, 1])
                for bad in (-1, V, 2 ** 31 - 1, -2 ** 31):
                    self.ids[g.random((M, k)) < 0.05] = bad
            if M > 4:
                self.ids[1] = -1
                self.t[2] = -np.inf
                self.t[3] = np.finfo(np.float32).min
        if kind == PR:
            self.t = np.exp(self.t) / np.exp(self.t).sum(1, keepdims=True).clip(1e-30) * 0.9
            self.t[np.isnan(self.t)] = 0
        self.ids, self.t = self.ids.astype(np.int32), self.t.astype(np.float32)
        self.dloss = g.normal(size=M).astype(np.float32)
        self.dev = to_dev_bf16(self.X), to_dev_bf16(self.W), to_dev(self.ids), to_dev(self.t)


def check_forward(P, c, tau, **out):
    lse, loss, z_top = P.lm_head_distill_fwd(*c.dev, temperature=tau, target=c.kind, **out)
    f = ld.forward(c.X, c.W, c.ids, c.t, tau, c.kind)
    for name, got in (("lse", lse), ("loss", loss), ("z_top", z_top)):
        err = np.abs(host(got).astype(np.float64) - f[name])
        # (a binary32 result carries its own rounding, inside each allowance but where it is zero)
        tol = f["tol_" + {"z_top": "z"}.get(name, name)] + 2.0 ** -24 * np.abs(f[name])
        assert (err <= tol).all(), "%s: %d of %d off, by up to %.3g of what is allowed" % (
            name, (err > tol).sum(), err.size, (err[err > tol] / np.maximum(tol[err > tol], 1e-300)).max())
    return f, lse, loss, z_top


def check_gradients(c, f, tau, dloss, grad_scale, dX, dW, add=None, what=""):
    mid, lo, hi = (f64(v) for v in ld.dz_band(f, tau, dloss, grad_scale))
    width = hi - lo
    x, w = f64(c.X), f64(c.W)
    if dX is not None:
        check_bf16(bf16_bits(dX), mid @ w, np.abs(mid) @ np.abs(w), what=what + " dX", slack=width @ np.abs(w))
    if dW is not None:
        ref, den, slack = mid.T @ x, np.abs(mid).T @ np.abs(x), width.T @ np.abs(x)
        if add is not None:
            ref, den = ref + add, den + np.abs(add)
        if "float32" in str(dW.dtype):
            check_fp32(host(dW), ref, den, what=what + " dW", slack=slack)
        else:
            check_bf16(bf16_bits(dW), ref, den, what=what + " dW", slack=slack)


SHAPES = [(1, 1, 8, 1), (1, 5, 8, 3), (3, 130, 16, 4), (77, 503, 40, 7), (129, 128, 128, 2), (128, 384, 256, 16),
          (255, 1000, 72, 70), (300, 257, 200, 33)]


@pytest.mark.parametrize("M,V,K,k", SHAPES)
@pytest.mark.parametrize("kind", [L, PR])
@pytest.mark.parametrize("tau", [1.0, 2.5])
def test_shapes(P, M, V, K, k, kind, tau):
    import torch
    c = Case(M + V + k, M, V, K, k, kind)
    f, lse, loss, z_top = check_forward(P, c, tau)
    saved = (*c.dev, lse, z_top)
    dX, dW = P.lm_head_distill_bwd(*saved, temperature=tau, target=kind)
    check_gradients(c, f, tau, np.ones(M), 1.0, dX, dW, what="%dx%dx%d" % (M, V, K))
    # per-row upstream gradients, scaled, dW in BF16
    bw = torch.empty(V, K, dtype=torch.bfloat16, device="cuda")
    dX, dW = P.lm_head_distill_bwd(*saved, temperature=tau, target=kind, dloss=to_dev(c.dloss), grad_scale=-0.25, dW=bw)
    assert dW is bw
    check_gradients(c, f, tau, c.dloss.astype(np.float64), -0.25, dX, dW, what="%dx%dx%d" % (M, V, K))


@pytest.mark.parametrize("M,V,K,k", [(65, 9000, 64, 20), (130, 8193, 40, 5), (33, 16384, 24, 9), (1, 20001, 16, 64)])
def test_wide_vocabularies(P, M, V, K, k):
    c = Case(V, M, V, K, k)
    c.ids[:, -1] = V - 1                                       # an entry in the last column
    c.ids[:, 0] = min(8191, V - 1)
    c.dev = c.dev[:2] + (to_dev(c.ids), c.dev[3])
    f, lse, loss, z_top = check_forward(P, c, 1.0)
    dX, dW = P.lm_head_distill_bwd(*c.dev, lse, z_top)
    check_gradients(c, f, 1.0, np.ones(M), 1.0, dX, dW)


# one tile of 128 x 128 a CU (256 of them) and one more, two a CU (512) and more, up to 128 rows and more of them
@pytest.mark.parametrize("M,V,K", [(129, 16384, 24), (257, 10900, 72), (128, 32769, 8), (255, 32768, 16), (256, 32769, 136),
                                   (100, 65601, 16)])
def test_tiles_of_the_forward(P, M, V, K):
    check_forward(P, Case(M + K, M, V, K, 6), 1.5)


# the same of the backward's logits: one tile a CU, two, and up to 128 rows of more
@pytest.mark.parametrize("M,V,K", [(255, 1000, 72), (300, 11000, 40), (513, 6500, 16), (128, 65601, 8)])
def test_tiles_of_the_backward(P, M, V, K):
    c = Case(M + V, M, V, K, 6)
    f, lse, loss, z_top = check_forward(P, c, 1.5)
    dX, dW = P.lm_head_distill_bwd(*c.dev, lse, z_top, temperature=1.5, dloss=to_dev(c.dloss))
    check_gradients(c, f, 1.5, c.dloss.astype(np.float64), 1.0, dX, dW)


def test_long_reduction(P):
    """A vocabulary and a size of dX whose product takes the large tiles, split over the vocabulary."""
    c = Case(15, 300, 33001, 1024, 8)
    f, lse, loss, z_top = check_forward(P, c, 1.0)
    dX, _ = P.lm_head_distill_bwd(*c.dev, lse, z_top, want_dw=False)
    check_gradients(c, f, 1.0, np.ones(300), 1.0, dX, None)


@pytest.mark.parametrize("M,V", [(16384, 90001), (30001, 131072)])
def test_several_chunks(P, M, V):
    """dz of more than 2.5 GiB: two and three chunks of the vocabulary, the last one ragged or whole. Sampled rows of
    the losses and dX, and rows of dW on both sides of every chunk's border (from the forward's lse, itself checked)."""
    import torch
    K, k = 16, 4
    c = Case(M, M, V, K, k, plain=True)
    lse, loss, z_top = P.lm_head_distill_fwd(*c.dev)
    dX, dW = P.lm_head_distill_bwd(*c.dev, lse, z_top, dloss=to_dev(c.dloss))
    rows = np.unique(np.r_[0, M - 1, np.random.default_rng(2).integers(0, M, 30)])
    f = ld.forward(c.X[rows], c.W, c.ids[rows], c.t[rows], 1.0, L)
    for name, got in (("lse", lse), ("loss", loss)):
        assert (np.abs(host(got)[rows] - f[name]) <= f["tol_" + name] + 2.0 ** -24 * np.abs(f[name])).all(), name
    part = Case(0, 1, 1, 8, 1)
    part.X, part.W = c.X[rows], c.W
    check_gradients(part, f, 1.0, c.dloss[rows].astype(np.float64), 1.0, dX[torch.from_numpy(rows).cuda()], None)
    chunks = -(-(M + 127) // 128 * 128 * ((V + 127) // 128 * 128) * 2 // (5 << 29))
    assert chunks >= 2
    width = (-(-(V + 127) // 128 * 128 // chunks) + 255) // 256 * 256
    cols = np.unique(np.r_[0, V - 1, [b + d for b in range(width, V, width) for d in (-1, 0)],
                           np.random.default_rng(3).integers(0, V, 12)])
    # dz of those columns and all rows: the columns as a vocabulary of their own, with the whole one's lse
    x, w = f64(c.X), f64(c.W[cols])
    a, S = x @ w.T, np.abs(x) @ np.abs(w).T
    place = np.full(V, -1, np.int64)
    place[cols] = np.arange(cols.size)
    q, _, tol_q = ld.teacher(c.ids, c.t, V, 1.0, L)
    at = place[c.ids]
    g = dict(a=a, tol_a=ld.TOL_Z * S, lse=host(lse).astype(np.float64), tol_lse=np.zeros(M), q=q, tol_q=tol_q,
             ok=np.ones_like(at, bool), at=at)
    # (entries elsewhere count for Q, but have no place here: a column of their own, dropped afterwards)
    g["at"] = np.where(at >= 0, at, cols.size)
    g["a"] = np.concatenate((a, np.zeros((M, 1))), 1)
    g["tol_a"] = np.concatenate((g["tol_a"], np.zeros((M, 1))), 1)
    mid, lo, hi = (f64(v)[:, :-1] for v in ld.dz_band(g, 1.0, c.dloss.astype(np.float64), 1.0))
    check_fp32(host(dW[torch.from_numpy(cols).cuda()]), mid.T @ x, np.abs(mid).T @ np.abs(x), what="dW columns",
               slack=(hi - lo).T @ np.abs(x))


@pytest.mark.parametrize("k", [1, 63, 64, 65, 200, 1024])
def test_numbers_of_entries(P, k):
    c = Case(k, 9, 1500, 32, k)
    f, lse, loss, z_top = check_forward(P, c, 0.5)
    dX, dW = P.lm_head_distill_bwd(*c.dev, lse, z_top, temperature=0.5)
    check_gradients(c, f, 0.5, np.ones(9), 1.0, dX, dW)


def test_one_of_the_gradients_and_accumulation(P):
    import torch
    c = Case(5, 40, 300, 64, 6)
    f, lse, loss, z_top = check_forward(P, c, 1.0)
    saved = (*c.dev, lse, z_top)
    dX, dW = P.lm_head_distill_bwd(*saved)
    a, none = P.lm_head_distill_bwd(*saved, want_dw=False)
    assert none is None and torch.equal(a, dX)
    none, b = P.lm_head_distill_bwd(*saved, want_dx=False)
    assert none is None and torch.equal(b, dW)
    g = np.random.default_rng(1).normal(size=(300, 64)).astype(np.float32)
    main = to_dev(g)
    P.lm_head_distill_bwd(*saved, dW=main, accumulate_dw=True)
    check_gradients(c, f, 1.0, np.ones(40), 1.0, None, main, add=g.astype(np.float64))


def test_agrees_with_the_cross_entropy(P):
    """One entry per row is the cross-entropy with that target: against puro_lm_head_ce_*."""
    import torch
    c = Case(6, 256, 640, 128, 1, plain=True)
    lse, loss, z_top = P.lm_head_distill_fwd(*c.dev)
    target = c.dev[2][:, 0].contiguous()
    lse2, loss2 = P.lm_head_ce_fwd(c.dev[0], c.dev[1], target)
    torch.testing.assert_close(lse, lse2, rtol=2e-6, atol=2e-6)
    torch.testing.assert_close(loss, loss2, rtol=1e-5, atol=1e-5)
    dX, dW = P.lm_head_distill_bwd(*c.dev, lse2, z_top)
    dX2, dW2 = P.lm_head_ce_bwd(c.dev[0], c.dev[1], target, lse2)
    # dz differs where the target's logit, taken twice, falls on the other side of a rounding
    step = 2.0 ** -8
    for a, b in ((dX, dX2), (dW, dW2)):
        assert float((a.float() - b.float()).norm() / b.float().norm()) < step


def test_padding_rows_change_nothing(P):
    """The rows of padding tokens (no entries) get zeros, the others what they get without them."""
    import torch
    c = Case(7, 96, 700, 64, 8, plain=True)
    lse, loss, z_top = P.lm_head_distill_fwd(*c.dev)
    dX, dW = P.lm_head_distill_bwd(*c.dev, lse, z_top)
    ids = c.dev[2].clone()
    ids[50:] = -1
    lse2, loss2, z2 = P.lm_head_distill_fwd(c.dev[0], c.dev[1], ids, c.dev[3])
    assert torch.equal(lse, lse2) and torch.equal(loss[:50], loss2[:50]) and not loss2[50:].any() and not z2[50:].any()
    dX2, dW2 = P.lm_head_distill_bwd(c.dev[0], c.dev[1], ids, c.dev[3], lse2, z2)
    assert torch.equal(dX[:50], dX2[:50]) and not dX2[50:].any()
    cut = [v[:50].contiguous() for v in (c.dev[0], ids, c.dev[3], lse, z_top)]
    _, dW3 = P.lm_head_distill_bwd(cut[0], c.dev[1], cut[1], cut[2], cut[3], cut[4])
    torch.testing.assert_close(dW2, dW3, rtol=0, atol=1e-5 * float(dW3.abs().max()))


@pytest.mark.parametrize("value", [float("nan"), float("inf")])
def test_padding_rows_may_hold_anything(P, value):
    """Hidden states of rows without a gradient (no entries, dloss 0, probabilities 0) are never part of one."""
    import torch
    c = Case(9, 150, 700, 72, 5, PR, plain=True)
    X, W, ids, t = c.dev
    ids[3], ids[140:] = -1, -1
    t[20] = 0
    dloss = to_dev(c.dloss)
    dloss[60:64] = 0
    idle = [3, 20, *range(60, 64), *range(140, 150)]
    lse, loss, z_top = P.lm_head_distill_fwd(X, W, ids, t, target=PR)
    want = P.lm_head_distill_bwd(X, W, ids, t, lse, z_top, target=PR, dloss=dloss)
    assert not want[0][idle].any()
    bad = X.clone()
    bad[idle] = value
    lse2, loss2, z2 = P.lm_head_distill_fwd(bad, W, ids, t, target=PR)
    empty = [3, 20, *range(140, 150)]
    assert torch.isfinite(loss2[empty]).all() and not loss2[empty].any()
    live = [i for i in range(150) if i not in idle]
    assert torch.equal(lse[live], lse2[live]) and torch.equal(loss[live], loss2[live]) and torch.equal(z_top[live], z2[live])
    got = P.lm_head_distill_bwd(bad, W, ids, t, lse2, z2, target=PR, dloss=dloss)
    assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])
    # a NaN upstream gradient reaches every value of its row, underflowed exponentials' too
    lse[7] += 1000
    dloss[7] = float("nan")
    assert torch.isnan(P.lm_head_distill_bwd(X, W, ids, t, lse, z_top, target=PR, dloss=dloss)[1]).all()


@pytest.mark.parametrize("kind,value", [(L, np.nan), (L, np.inf), (PR, np.nan)])
def test_special_values_stay_in_their_row(P, kind, value):
    import torch
    c = Case(8, 20, 300, 32, 70, kind, plain=True)
    want = P.lm_head_distill_fwd(*c.dev, target=kind)
    want_dx = P.lm_head_distill_bwd(*c.dev, want[0], want[2], target=kind, want_dw=False)[0]
    t = c.dev[3].clone()
    t[4, 66] = value
    got = P.lm_head_distill_fwd(c.dev[0], c.dev[1], c.dev[2], t, target=kind)
    assert torch.equal(got[0], want[0]) and torch.equal(got[2], want[2])
    others = [i for i in range(20) if i != 4]
    assert torch.isnan(got[1][4]) and torch.equal(got[1][others], want[1][others])
    dX = P.lm_head_distill_bwd(c.dev[0], c.dev[1], c.dev[2], t, got[0], got[2], target=kind, want_dw=False)[0]
    assert torch.isnan(dX[4]).all() and torch.equal(dX[others], want_dx[others])
    # the same among the entries that do not count: nothing
    ids = c.dev[2].clone()
    ids[4, 66] = -1
    a = P.lm_head_distill_fwd(c.dev[0], c.dev[1], ids, t, target=kind)
    assert torch.isfinite(a[1]).all()
    # a row of nothing but NaN
    t[4] = float("nan")
    assert torch.isnan(P.lm_head_distill_fwd(c.dev[0], c.dev[1], c.dev[2], t, target=kind)[1][4])


@pytest.mark.parametrize("shift", [-300.0, 250.0])
def test_far_logits(P, shift):
    """Logits far from zero: the columns past the vocabulary (whose product is 0) must not reach the sums, nor their
    gradient (e^300 overflows) the others'."""
    c = Case(9, 40, 333, 64, 5, plain=True)
    x, w = f64(c.X), f64(c.W)
    x[:, 0], w[:, 0] = 16.0, shift / 16.0
    c.X, c.W = bf16.from_f64_rne(x), bf16.from_f64_rne(w)
    c.dev = (to_dev_bf16(c.X), to_dev_bf16(c.W)) + c.dev[2:]
    f, lse, loss, z_top = check_forward(P, c, 1.0)
    dX, dW = P.lm_head_distill_bwd(*c.dev, lse, z_top)
    check_gradients(c, f, 1.0, np.ones(40), 1.0, dX, dW)


def test_empty(P):
    import torch
    c = Case(10, 0, 64, 16, 3)
    lse, loss, z_top = P.lm_head_distill_fwd(*c.dev)
    assert lse.shape == (0,) and z_top.shape == (0, 3)
    for dt in (torch.float32, torch.bfloat16):
        dW = torch.full((64, 16), 3.0, dtype=dt, device="cuda")
        P.lm_head_distill_bwd(*c.dev, lse, z_top, dW=dW)
        assert not dW.any()
    dW = torch.full((64, 16), 3.0, device="cuda")
    P.lm_head_distill_bwd(*c.dev, lse, z_top, dW=dW, accumulate_dw=True)
    assert (dW == 3).all()


def test_same_bytes_every_time(P):
    import torch
    c = Case(11, 300, 9001, 64, 40)
    runs = []
    for _ in range(3):
        lse, loss, z_top = P.lm_head_distill_fwd(*c.dev)
        runs.append((lse, loss, z_top, *P.lm_head_distill_bwd(*c.dev, lse, z_top)))
    for r in runs[1:]:
        assert all(torch.equal(a, b) for a, b in zip(runs[0], r))


def test_graph_replays(P):
    """Captured and replayed on changed inputs, eager calls in between; outputs and workspaces of their own."""
    import torch
    c = Case(12, 140, 600, 64, 6, plain=True)
    X, W, ids, t = (v.clone() for v in c.dev)

    def step():
        lse, loss, z_top = P.lm_head_distill_fwd(X, W, ids, t, temperature=2.0)
        return (lse, loss, z_top, *P.lm_head_distill_bwd(X, W, ids, t, lse, z_top, temperature=2.0))

    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        step()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=s):
            kept = step()
    torch.cuda.current_stream().wait_stream(s)
    for n in range(4):
        X.copy_(c.dev[0].roll(n, 0))
        ids.copy_(c.dev[2].roll(n, 1))
        want = step()
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(kept, want))


def test_autograd(P):
    import torch
    c = Case(13, 50, 400, 64, 6)
    f = ld.forward(c.X, c.W, c.ids, c.t, 2.0, L)
    for main in (False, True):
        X, W = c.dev[0].clone().requires_grad_(True), torch.nn.Parameter(c.dev[1].clone())
        if main:
            W.main_grad = torch.zeros(400, 64, device="cuda")
        loss = P.lm_head_distill(X, W, c.dev[2], c.dev[3], 2.0)
        weights = to_dev(c.dloss)
        (loss * weights).sum().backward()
        check_gradients(c, f, 2.0, c.dloss.astype(np.float64), 1.0, X.grad, W.main_grad if main else W.grad)
        assert (W.grad is None) == main
    X = c.dev[0].clone()                                       # no gradient of the hidden states
    W = torch.nn.Parameter(c.dev[1].clone())
    P.lm_head_distill(X, W, c.dev[2], c.dev[3], 2.0).mean().backward()
    assert W.grad is not None


def test_refusals(P):
    import torch
    c = Case(14, 16, 64, 16, 3)
    X, W, ids, t = c.dev
    f = P.lm_head_distill_fwd
    for bad in ((X.float(), W, ids, t), (X, W, ids.long(), t), (X, W, ids, t.double()), (X, W, ids, t.bfloat16())):
        with pytest.raises(TypeError):
            f(*bad)
    for bad in ((X[:, :8], W, ids, t), (X, W[:, :8], ids, t), (X, W, ids[:8], t), (X, W, ids, t[:, :2]),
                (X.cpu(), W, ids, t), (X, W, ids[:, 0], t)):
        with pytest.raises(ValueError):
            f(*bad)
    for args, code in ((dict(temperature=0.0), 3), (dict(temperature=float("nan")), 3), (dict(target=2), 3)):
        with pytest.raises(P.PuroError) as e:
            f(X, W, ids, t, **args)
        assert e.value.code == code
    lse, loss, z_top = f(X, W, ids, t)
    with pytest.raises(P.PuroError) as e:                       # a BF16 sum would lose what it adds
        P.lm_head_distill_bwd(X, W, ids, t, lse, z_top, dW=torch.zeros_like(W), accumulate_dw=True)
    assert e.value.code == 3
    with pytest.raises(ValueError):
        P.lm_head_distill_bwd(X, W, ids, t, lse, z_top, dloss=torch.ones(15, device="cuda"))
    with pytest.raises(AssertionError):
        f(X, W, ids, t, ws=torch.empty(16, dtype=torch.uint8, device="cuda"))
