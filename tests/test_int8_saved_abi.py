"""Host-side checks of the int8 linear layer's saved copies (no GPU): either of
them, with its scales, may be left out where the gradient that reads it is not
wanted."""

import ctypes

import pytest

from test_abi import ERR_NULL, ERR_WORKSPACE, FAKE, puro  # noqa: F401

BIG = 1 << 50
X_ALONE, W_ALONE = (FAKE, FAKE, None, None), (None, None, FAKE, FAKE)


@pytest.mark.parametrize("there", [X_ALONE, W_ALONE, (None,) * 4])
def test_forward(puro, there):  # noqa: F811
    f = puro.lib().puro_int8_linear_fwd
    # (accepted: the workspace's size is the next thing looked at)
    assert f(FAKE, FAKE, 13, 32, 48, FAKE, ctypes.byref(puro.Saved(*there)), FAKE, 0, None) == ERR_WORKSPACE


@pytest.mark.parametrize("there,dX,dW,status", [
    (W_ALONE, FAKE, None, ERR_WORKSPACE), (X_ALONE, None, FAKE, ERR_WORKSPACE), (W_ALONE, None, FAKE, ERR_NULL),
    (X_ALONE, FAKE, None, ERR_NULL), (W_ALONE, FAKE, FAKE, ERR_NULL), (X_ALONE, FAKE, FAKE, ERR_NULL),
    ((None,) * 4, FAKE, None, ERR_NULL), ((FAKE, None, FAKE, FAKE), FAKE, None, ERR_NULL), ((FAKE, FAKE, None, FAKE), None, FAKE, ERR_NULL)])
def test_backward(puro, there, dX, dW, status):  # noqa: F811
    f = puro.lib().puro_int8_linear_bwd
    assert f(FAKE, ctypes.byref(puro.Saved(*there)), 13, 32, 48, dX, dW, 0, FAKE, 0, None) == status
