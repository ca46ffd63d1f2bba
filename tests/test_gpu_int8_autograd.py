"""The int8 linear layer as an autograd operation: its gradients against central
differences of its own outputs, forward mode."""

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
