"""The int8 linear layer and quantisers without channels: sums of nothing are 0
and scales of nothing 1, whatever the workspace held before."""

import numpy as np
import pytest

from oracle import bf16

from gpu_util import to_dev_bf16

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def P():
    from paper_2608_27370_amd import puro
    puro.lib()
    return puro


@pytest.mark.parametrize("want_saved", [True, False])
@pytest.mark.parametrize("M,N", [(1, 16), (13, 32), (100, 208), (300, 2048)])
def test_a_layer_without_input_channels(P, M, N, want_saved):
    import torch
    X, W = (torch.empty(n, 0, dtype=torch.bfloat16, device="cuda") for n in (M, N))
    for byte in (0xFF, 0x7F):                                    # NaN and large numbers, as binary32 reads them
        ws = torch.full((1 << 20,), byte, dtype=torch.uint8, device="cuda")
        Y = torch.full((M, N), 7.0, dtype=torch.bfloat16, device="cuda")
        P.int8_linear_fwd(X, W, Y=Y, want_saved=want_saved, ws=ws)
        assert not Y.view(torch.int16).any().item()              # +0 everywhere
    y, saved = P.int8_linear_fwd(X, W)
    dX, dW = P.int8_linear_bwd(Y, saved)
    assert not y.any().item() and dX.shape == (M, 0) and dW.shape == (N, 0)


def test_the_autograd_operation_without_input_channels(P):
    import torch
    X = torch.zeros(2, 3, 0, dtype=torch.bfloat16, device="cuda", requires_grad=True)
    W = torch.zeros(32, 0, dtype=torch.bfloat16, device="cuda", requires_grad=True)
    Y = P.int8_linear(X, W)
    assert Y.shape == (2, 3, 32) and not Y.detach().any().item()
    Y.backward(torch.ones_like(Y))
    assert X.grad.shape == X.shape and W.grad.shape == W.shape
    with torch.no_grad():
        assert not P.int8_linear(X, W).any().item()


def test_scales_of_rows_without_columns(P):
    """1 (as of rows of zeros), new ones and given ones, whatever the memory held."""
    import torch
    nan = torch.full((1 << 16,), float("nan"), device="cuda")
    del nan                                                      # (its memory is what the next call's outputs take)
    gu = torch.empty(5, 0, dtype=torch.bfloat16, device="cuda")
    r = P.swiglu_quantize_int8(gu, 0)
    assert r["q"].shape == (5, 0) and (r["scale"] == 1).all().item()
    given = torch.full((5,), float("nan"), device="cuda")
    assert P.swiglu_quantize_int8(gu, 0, out=dict(scale=given))["scale"] is given and (given == 1).all().item()
    given.fill_(float("nan"))
    P.quantize_int8(gu, out=dict(scale=given))
    assert (given == 1).all().item()
