"""RMSNorm encoded to int8 where rows are tiny and eps does not hide it: their
squares lose bits in binary32 below 2^-126 and vanish below 2^-149, the codes and
scales are those of any other row (oracle/int8.py's bands)."""

import numpy as np
import pytest

from oracle import bf16, int8

from test_gpu_int8 import P, check_band, f64  # noqa: F401

from gpu_util import host, to_dev_bf16

pytestmark = pytest.mark.gpu

ROWS = [-1, -30, -48, -50, -52, -63, -70, -74, -75, -80, -100, -120, -126, -130]


def rows(C):
    """A row about each power of two of ROWS, as BF16 holds it (subnormal ones at the end), one of zeros between."""
    g = np.random.default_rng(C)
    x = g.normal(size=(len(ROWS), C)) * 2.0 ** np.array(ROWS)[:, None]
    x[:, 0] = 2.0 ** np.array(ROWS)                              # (none is all zeros)
    return bf16.from_f64_rne(x)


# a block a row (the longest in more than its registers), a wave, 16 lanes
@pytest.mark.parametrize("R,C", [(1, 16), (1, 128), (1, 1536), (1, 2064), (1, 24592), (74, 1536), (74, 512), (293, 128), (293, 16)])
@pytest.mark.parametrize("eps", [0.0, 2.0 ** -149, 2.0 ** -120, 2.0 ** -101, 2.0 ** -100, 2.0 ** -60])
def test_tiny_rows_are_normalised_as_others(P, R, C, eps):  # noqa: F811
    x = np.tile(rows(C), (R, 1))
    gamma = bf16.from_f64_rne(1 + 0.3 * np.random.default_rng(1).normal(size=C))
    r = P.rmsnorm_quantize_int8(to_dev_bf16(x), to_dev_bf16(gamma), eps, want_rstd=True)
    y, rstd, e = int8.rmsnorm(f64(x), f64(gamma), eps)
    check_band(r["q"], r["scale"], y, e, "C %d eps %g" % (C, eps))
    got = host(r["rstd"]).astype(np.float64)
    fits = rstd < 2.0 ** 127.5                                   # (beyond binary32's largest number: infinity)
    assert (np.abs(got - rstd)[fits] <= e * rstd[fits]).all()
    assert np.isinf(got[rstd > 2.0 ** 128]).all()


def test_a_row_of_zeros_without_eps_has_no_norm(P):  # noqa: F811
    x = rows(128)
    x[3] = 0
    ones = to_dev_bf16(bf16.from_f64_rne(np.ones(128)))
    r = P.rmsnorm_quantize_int8(to_dev_bf16(x), ones, 0.0, want_rstd=True)
    s = host(r["scale"])
    assert np.isnan(s[3]) and not host(r["q"])[3].any() and np.isfinite(np.delete(s, 3)).all()
    assert np.isinf(host(r["rstd"])[3])
    s = host(P.rmsnorm_quantize_int8(to_dev_bf16(x), ones, 2.0 ** -149)["scale"])
    assert s[3] == 1.0 and np.isfinite(s).all()
