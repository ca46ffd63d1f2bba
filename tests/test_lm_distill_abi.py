"""Host-side refusals of the distillation calls (no GPU): each invalid
argument returns its documented status before anything is launched."""

import pytest

from test_abi import ERR_ALIGN, ERR_NULL, ERR_SHAPE, ERR_UNSUPPORTED, ERR_WORKSPACE, FAKE, OK, puro  # noqa: F401

BIG = 1 << 50


@pytest.fixture(scope="module")
def call(puro):  # noqa: F811
    L = puro.lib()

    def call(bwd, X=FAKE, W=FAKE, ids=FAKE, t=FAKE, M=100, V=500, K=64, k=8, kind=0, tau=1.0, lse=FAKE, loss=FAKE, z=FAKE,
             dloss=None, g=1.0, dX=FAKE, dW=FAKE, out=1, acc=0, ws=FAKE, nb=BIG):
        if bwd:
            return L.puro_lm_head_distill_bwd(X, W, ids, t, lse, z, M, V, K, k, kind, tau, dloss, g, dX, dW, out, acc, ws,
                                              nb, None)
        return L.puro_lm_head_distill_fwd(X, W, ids, t, M, V, K, k, kind, tau, lse, loss, z, ws, nb, None)
    return call


@pytest.mark.parametrize("bwd", [False, True])
def test_refusals_of_both_passes(call, puro, bwd):  # noqa: F811
    f = lambda **a: call(bwd, **a)
    assert f(M=-1) == f(V=0) == f(K=0) == f(M=(1 << 21) + 1) == f(V=(1 << 21) + 1) == f(K=(1 << 21) + 8) == ERR_SHAPE
    assert f(k=0) == f(k=1025) == ERR_SHAPE
    assert f(K=60) == ERR_ALIGN
    assert f(kind=2) == ERR_UNSUPPORTED
    for tau in (0.0, -1.0, float("nan"), float("inf"), 1e-40, 3e38):
        assert f(tau=tau) == ERR_UNSUPPORTED
    for n in ("X", "W", "ids", "t", "lse", "z", "ws"):
        assert f(**{n: None}) == ERR_NULL, n
    for n in ("X", "W", "ws"):
        assert f(**{n: FAKE + 8}) == ERR_ALIGN, n
    for n in ("ids", "t", "lse", "z"):
        assert f(**{n: FAKE + 2}) == ERR_ALIGN, n
    need = puro.lib().puro_lm_head_distill_workspace_size(100, 500, 64, 8, int(bwd))
    assert need > 0 and f(nb=need - 1) == ERR_WORKSPACE


def test_refusals_of_one_pass(call):
    assert call(False, loss=None) == ERR_NULL
    assert call(False, loss=FAKE + 2) == ERR_ALIGN
    f = lambda **a: call(True, **a)
    assert f(g=float("nan")) == f(g=float("inf")) == f(out=2) == f(out=0, acc=1) == ERR_UNSUPPORTED
    assert f(dX=FAKE + 8) == f(dW=FAKE + 8) == f(dloss=FAKE + 2) == ERR_ALIGN


def test_sizes_and_empty_calls(call, puro):  # noqa: F811
    size = puro.lib().puro_lm_head_distill_workspace_size
    for bad in ((-1, 5, 8, 1, 0), (0, 5, 8, 1, 1), (4, 0, 8, 1, 1), (4, 5, 12, 1, 1), (4, 5, 8, 0, 1)):
        assert size(*bad) == 0
    assert size(4, 5, 8, 1, 1) > size(4, 5, 8, 1, 0) > 0
    assert call(False, M=0, X=None, ids=None, t=None, lse=None, loss=None, z=None, ws=None, nb=0) == OK
    assert call(True, dX=None, dW=None) == OK                  # neither gradient is wanted
    assert call(True, M=0, dW=None, X=None, ids=None, t=None, lse=None, z=None, ws=None, nb=0) == OK
