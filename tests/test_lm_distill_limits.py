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
