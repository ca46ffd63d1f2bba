"""The sizes that the distillation calls take (no GPU): what a launch cannot
hold is refused before anything is launched, the largest sizes below it are
not."""

import pytest

from test_abi import ERR_SHAPE, ERR_WORKSPACE, FAKE, puro  # noqa: F401


@pytest.mark.parametrize("bwd", [False, True])
@pytest.mark.parametrize("M,V", [(1 << 21, (1 << 18) + 1), ((1 << 18) + 1, 1 << 21), (1 << 21, 1 << 21)])
def test_more_logits_than_a_launch_takes(puro, bwd, M, V):  # noqa: F811
    """2^24 tiles of 256 x 256 logits are 2^32 threads, more than a launch holds: half as many are the limit."""
    L = puro.lib()
    size, k, K = L.puro_lm_head_distill_workspace_size, 1, 8

    def call(M, V):
        if bwd:
            return L.puro_lm_head_distill_bwd(FAKE, FAKE, FAKE, FAKE, FAKE, FAKE, M, V, K, k, 0, 1.0, None, 1.0, FAKE, FAKE, 1, 0,
                                              FAKE, 16, None)
        return L.puro_lm_head_distill_fwd(FAKE, FAKE, FAKE, FAKE, M, V, K, k, 0, 1.0, FAKE, FAKE, FAKE, FAKE, 16, None)

    assert call(M, V) == ERR_SHAPE and size(M, V, K, k, int(bwd)) == 0
    for m, v in ((1 << 21, 1 << 18), (1 << 18, 1 << 21)):
        assert call(m, v) == ERR_WORKSPACE and size(m, v, K, k, int(bwd)) > 16


@pytest.mark.parametrize("M,V", [(1 << 21, 151936), (1 << 21, 1 << 18), (1900000, 50257), (300001, 151936), (8192, 151936),
                                 (16384, 90001), (20000, 67200), (1, 1 << 21)])
def test_copies_of_the_gradient_within_what_is_stated(puro, M, V):  # noqa: F811
    """The backward's workspace holds two copies of dz of at most 2.5 GiB each, beside what its other parts take
    (padded to 128 rows): a factor a row, a value an entry, the transposed X and W, dX in binary32, and the partial sums
    of dX and dW at one unit of 256 x 256 values per compute unit, with 1 MiB for the paddings of each part."""
    K, k = 8, 1
    Mp, Vp = (M + 127) // 128 * 128, (V + 127) // 128 * 128
    rest = 4 * Mp + 4 * M * k + 2 * Mp * K + 2 * Vp * K + 4 * M * K + 256 * 256 * 256 * 4 + (1 << 20)
    used = puro.lib().puro_lm_head_distill_workspace_size(M, V, K, k, 1)
    assert used <= 2 * min(5 << 29, 2 * Mp * Vp) + rest


def test_factors_of_the_gradient(puro):  # noqa: F811
    """grad_scale and its quotient by the temperature are finite: times a dloss of 0 they have to be 0."""
    from test_abi import ERR_UNSUPPORTED

    def f(g, tau):
        return puro.lib().puro_lm_head_distill_bwd(FAKE, FAKE, FAKE, FAKE, FAKE, FAKE, 100, 500, 64, 8, 0, tau, None, g, FAKE, FAKE,
                                                   1, 0, FAKE, 16, None)

    for g, tau in ((1e3, 1e-37), (-1e3, 1e-37), (3e38, 0.5), (float("nan"), 1.0), (float("inf"), 1e10)):
        assert f(g, tau) == ERR_UNSUPPORTED
    for g, tau in ((1.0, 1e-37), (3e38, 2.0), (0.0, 1e-37), (1e-38, 1e10)):
        assert f(g, tau) == ERR_WORKSPACE
