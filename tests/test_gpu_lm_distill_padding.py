"""Padding tokens of the distillation loss: rows without entries (or whose
weights are all 0) have no gradient, whatever their hidden state and their
upstream gradient hold."""

import numpy as np
import pytest

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("value", [float("nan"), float("inf"), -3e38])
@pytest.mark.parametrize("target", ["logits", "probs"])
@pytest.mark.parametrize("M,V,K", [(40, 300, 64), (300, 4000, 72)])
def test_upstream_gradients_of_padding_tokens(value, target, M, V, K):
    import torch
    from paper_2608_27370_amd import puro as P
    g = torch.Generator(device="cuda").manual_seed(M)
    X = torch.randn(M, K, generator=g, device="cuda").to(torch.bfloat16)
    W = (torch.randn(V, K, generator=g, device="cuda") * 0.1).to(torch.bfloat16)
    ids = torch.randint(0, V, (M, 5), generator=g, device="cuda", dtype=torch.int32)
    t = torch.rand(M, 5, generator=g, device="cuda")
    kind = P.DISTILL_LOGITS if target == "logits" else P.DISTILL_PROBS
    pad = [0, 7, *range(M - 9, M)]
    ids[pad] = -1
    if target == "probs":
        ids[9] = 1
        t[9] = 0
        pad.append(9)
    dloss = torch.rand(M, generator=g, device="cuda")
    dloss[pad] = 0
    args = X, W, ids, t
    lse, loss, z_top = P.lm_head_distill_fwd(*args, temperature=0.5, target=kind)
    want = P.lm_head_distill_bwd(*args, lse, z_top, temperature=0.5, target=kind, dloss=dloss, grad_scale=4.0)
    bad = dloss.clone()
    bad[pad] = value
    got = P.lm_head_distill_bwd(*args, lse, z_top, temperature=0.5, target=kind, dloss=bad, grad_scale=4.0)
    assert not got[0][pad].any()
    assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])
    assert np.isfinite(got[1].cpu().numpy()).all()
