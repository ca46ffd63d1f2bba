"""The int8 linear layer as an autograd operation: its gradients against central
differences of its own outputs, what it keeps for a backward, forward mode."""

import numpy as np
import pytest

from gpu_util import to_dev

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def P():
    from paper_2608_27370_amd import puro
    puro.lib()
    return puro


def bf16(a):
    import torch
    return to_dev(np.asarray(a, np.float32)).to(torch.bfloat16)


def whole_numbers(seed, M, N, K):
    """X, W and dY whose codes are their values (or, where a scale is not 1, exact all the same): small whole numbers,
    and in every row and column that is quantised a 127 where it meets nothing but zeros of the other factor."""
    g = np.random.default_rng(seed)
    X, W, dY = (g.integers(-1, 2, s) for s in ((M, K), (N, K), (M, N)))
    X[:, 0], W[:, 0] = 127, 0                                    # X's rows
    W[:, 1], X[:, 1] = 127, 0                                    # W's rows
    dY[:, 0], W[0] = 127, 0                                      # dY's rows
    dY[0], X[0] = 127, 0                                         # dY's columns
    X[M - 1], dY[M - 1] = 127, 0                                 # X's columns
    W[N - 1], dY[:, N - 1] = 127, 0                              # W's columns
    return X, W, dY


@pytest.mark.parametrize("M,N,K", [(5, 16, 16), (40, 48, 64), (70, 64, 80)])
def test_gradients_are_the_differences_of_the_outputs(P, M, N, K):
    """The layer is bilinear in codes, and these inputs' codes are exact, as are theirs a step to either side: outputs of
    up to 256 lose nothing in BF16, so that central differences of sum(dY Y) with a step of 1 are the gradients exactly."""
    import torch
    X, W, dY = whole_numbers(M, M, N, K)

    def loss(x, w):
        with torch.no_grad():
            y = P.int8_linear(bf16(x), bf16(w)).double().cpu().numpy()
        live = dY != 0
        assert np.array_equal(y[live], (x @ w.T)[live])
        return float((dY * y)[live].sum())
    x, w = bf16(X).requires_grad_(), bf16(W).requires_grad_()
    P.int8_linear(x, w).backward(bf16(dY))
    g = np.random.default_rng(9)
    for grad, at, rows, cols in ((x.grad, 0, range(1, M - 1), range(2, K)), (w.grad, 1, range(1, N - 1), range(2, K))):
        grad = grad.double().cpu().numpy()
        for _ in range(12):
            r, c = int(g.choice(rows)), int(g.choice(cols))
            e = np.zeros_like((X, W)[at])
            e[r, c] = 1
            up, down = (loss(X + s * e, W) if at == 0 else loss(X, W + s * e) for s in (1, -1))
            assert grad[r, c] == (up - down) / 2, (at, r, c)


def test_forward_mode_is_refused(P):
    """Where nothing requires a gradient too, with gradients on and off: a tangent is not lost in silence."""
    import torch
    import torch.autograd.forward_ad as fwAD
    g = np.random.default_rng(1)
    X, W = bf16(g.normal(size=(3, 32))), bf16(g.normal(size=(16, 32)))
    with fwAD.dual_level():
        for x, w in ((fwAD.make_dual(X, torch.ones_like(X)), W), (X, fwAD.make_dual(W, torch.ones_like(W)))):
            with pytest.raises((NotImplementedError, RuntimeError)):
                P.int8_linear(x, w)
            with torch.no_grad(), pytest.raises((NotImplementedError, RuntimeError)):
                P.int8_linear(x, w)
    assert not P.int8_linear(X, W).requires_grad


def test_what_is_kept_is_what_the_backward_reads(P, monkeypatch):
    import torch
    g = np.random.default_rng(2)
    M, N, K = 37, 48, 64
    X, W, dY = bf16(g.normal(size=(M, K))), bf16(g.normal(size=(N, K))), bf16(g.normal(size=(M, N)))
    made, forward = [], P.int8_linear_fwd

    def recorded(*a, **kw):
        y, saved = forward(*a, **kw)
        made.append(saved)
        return y, saved
    monkeypatch.setattr(P, "int8_linear_fwd", recorded)

    def call(want_x, want_w):
        x, w = X.clone().requires_grad_(want_x), W.clone().requires_grad_(want_w)
        Y = P.int8_linear(x, w)
        if Y.requires_grad:
            Y.backward(dY)
        return Y.detach(), x.grad, w.grad, made[-1]
    Y, dX, dW, both = call(True, True)
    assert all(v is not None for v in both.values())
    for want_x, want_w in ((True, False), (False, True), (False, False)):
        y, dx, dw, kept = call(want_x, want_w)
        assert torch.equal(y, Y)
        assert dx is None or torch.equal(dx, dX)
        assert dw is None or torch.equal(dw, dW)
        assert (dx is not None, dw is not None) == (want_x, want_w)
        kept = kept or {}
        assert (kept.get("wq_t") is not None, kept.get("w_scale") is not None) == (want_x, want_x)
        assert (kept.get("xq_t") is not None, kept.get("x_scale") is not None) == (want_w, want_w)
    with torch.no_grad():
        assert torch.equal(P.int8_linear(X.requires_grad_(), W.requires_grad_()), Y) and not made[-1]


@pytest.mark.parametrize("M,N,K", [(1, 16, 32), (333, 512, 272), (0, 16, 16)])
def test_one_of_the_copies_alone(P, M, N, K):
    """Each gradient from the copy that it reads, bit for bit; without that copy it is refused."""
    import torch
    g = np.random.default_rng(M)
    X, W, dY = bf16(g.normal(size=(M, K))), bf16(g.normal(size=(N, K))), bf16(g.normal(size=(M, N)))
    Y, saved = P.int8_linear_fwd(X, W)
    dX, dW = P.int8_linear_bwd(dY, saved)
    y, for_dx = P.int8_linear_fwd(X, W, want_dw=False)
    z, for_dw = P.int8_linear_fwd(X, W, want_dx=False)
    none, nothing = P.int8_linear_fwd(X, W, want_dx=False, want_dw=False)
    assert torch.equal(y, Y) and torch.equal(z, Y) and torch.equal(none, Y) and not any(v is not None for v in nothing.values())
    if M:
        for part, names in ((for_dx, ("wq_t", "w_scale")), (for_dw, ("xq_t", "x_scale"))):
            assert {k for k, v in part.items() if v is not None} == set(names)
            assert all(torch.equal(part[k], saved[k]) for k in names)
    assert torch.equal(P.int8_linear_bwd(dY, for_dx, want_dw=False)[0], dX)
    assert torch.equal(P.int8_linear_bwd(dY, for_dw, want_dx=False)[1], dW)
    for part in (for_dx, for_dw, nothing):
        with pytest.raises(ValueError):
            P.int8_linear_bwd(dY, part)
