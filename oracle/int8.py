"""8-bit integer codes of rows and columns, and the product of such codes, in
float64 and exact integers.

Test infrastructure only (see the package docstring). A row x with amax = max |x|:

    s = fl32(amax / 127), r = fl32(127 / amax) (of unlimited exponent), code = the
    integer nearest to x r, ties to even; amax = 0: s = 1, codes 0; a NaN or an
    infinity among x: s = NaN, codes 0.

The paper states no integer format (it trains in FP8, Section 3.2): parity
unpinned; tests/test_oracle_int8.py pins it by exact rational arithmetic.

Bands of the fused forms, which encode a binary32 value without rounding it to
BF16 (u = 2^-24): a value known to a relative e moves v = 127 x / amax by 2 e |v|
(its own error and amax's), r and the product by 2 u |v| more; the codes of both
ends of that band are accepted, and s within e + 2 u.

  * RMSNorm: a lane sums whole chunks of 8 squares, fused, and the row's lanes are
    added up, all positive. Rows of up to 2048 values lie on 16 lanes (one chunk, 4
    additions more), a wave (8 ceil(cols / 512) terms and 6) or four waves (one chunk
    and 8), longer ones on four waves (8 ceil(cols / 2048) and 8): n roundings at most,
    halved by the root; the mean's division, eps's sum, root, reciprocal and two
    products at most 6 more: e = (n / 2 + 6) u.
  * SwiGLU: oracle/swiglu.py's 2^-20.
"""

import numpy as np

U = 2.0 ** -24


def _rows(x):
    x = np.asarray(x, dtype=np.float64)
    amax = np.abs(x).max(axis=1) if x.shape[1] else np.zeros(x.shape[0])
    bad = ~np.isfinite(amax)
    return x, np.where(bad, 0.0, amax), bad


def factor(amax):
    """r = fl32(127 / amax) of unlimited exponent, float64 (1 where amax is 0)."""
    a = np.where(amax > 0, amax, 127.0)
    up = np.where(a < 2.0 ** -100, 2.0 ** 64, 1.0)
    return (127.0 / (a * up)).astype(np.float32).astype(np.float64) * up


def encode_rows(x):
    """(codes int8 [R, C], scale float32 [R]) of the values x (exact in float64)."""
    x, amax, bad = _rows(x)
    with np.errstate(invalid="ignore"):
        q = np.where(bad[:, None], 0.0, np.rint(np.where(bad[:, None], 0.0, x) * factor(amax)[:, None]))
    s = np.where(bad, np.nan, np.where(amax > 0, amax / 127.0, 1.0)).astype(np.float32)
    return q.astype(np.int8), s


def encode_cols(x):
    """(codes [C, R rounded up to 16] with zeros behind the rows, scale [C])."""
    q, s = encode_rows(np.asarray(x).T)
    out = np.zeros((q.shape[0], -(-q.shape[1] // 16) * 16), np.int8)
    out[:, :q.shape[1]] = q
    return out, s


def band_rows(x, e):
    """(lowest codes, highest codes, scale, allowance of the scale) of values known to a relative e."""
    x, amax, bad = _rows(x)
    assert not bad.any()
    v = x * np.where(amax > 0, 127.0 / np.where(amax > 0, amax, 1.0), 0.0)[:, None]
    d = np.abs(v) * (2.0 * e + 2.0 * U)
    s = np.where(amax > 0, amax / 127.0, 1.0)
    return np.rint(v - d), np.rint(v + d), s, s * (e + 2.0 * U)


def rmsnorm(x, gamma, eps):
    """(y, rstd, relative allowance of y) of float64 x [R, C]."""
    rstd = 1.0 / np.sqrt((x * x).mean(axis=1) + eps)
    cols = x.shape[1]
    n = max(8 * -(-cols // 512) + 6, 16) if cols <= 2048 else 8 * -(-cols // 2048) + 8
    return x * rstd[:, None] * gamma, rstd, (n / 2.0 + 6.0) * U


def swiglu(gu):
    """(h, relative allowance) of float64 gu [R, 2 C]."""
    g, u = np.split(gu, 2, axis=1)
    with np.errstate(over="ignore"):                 # (a far negative gate: 0)
        return g / (1.0 + np.exp(-g)) * u, 2.0 ** -20


def gemm(A, sa, B, sb, bias=None, residual=None, add=None):
    """(D, allowance of a binary32 evaluation), float64: the sum, exact, rounded once (u), two products (u each) and a
    rounding of each sum that follows."""
    with np.errstate(invalid="ignore"):
        d = (A.astype(np.float64) @ B.astype(np.float64).T) * sa.astype(np.float64)[:, None] * sb.astype(np.float64)[None, :]
    tol = 3.01 * U * np.abs(d)
    for t in (bias, residual, add):
        if t is not None:
            d = d + t
            tol = tol + U * (np.abs(d) + tol)
    return d, tol + 2.0 ** -140
