"""The distillation calls at sizes whose element passes have more pieces than a
launch has threads."""

import pytest

pytestmark = pytest.mark.gpu


def test_clearing_a_gradient_of_64_gib():
    """M = 0: dW [2^21, 2^13] in FP32 is 2^32 pieces of 16 bytes."""
    import torch
    from paper_2608_27370_amd import puro as P
    V, K = 1 << 21, 1 << 13
    dW = torch.empty(V, K, dtype=torch.float32, device="cuda")
    try:
        for part in dW.split(1 << 17):
            part.fill_(3.0)
        assert P.lib().puro_lm_head_distill_bwd(None, None, None, None, None, None, 0, V, K, 1, 0, 1.0, None, 1.0, None,
                                                dW.data_ptr(), 1, 0, None, 0, P._stream()) == 0
        assert not any(bool(part.any()) for part in dW.split(1 << 15))
    finally:
        del dW
        torch.cuda.empty_cache()
