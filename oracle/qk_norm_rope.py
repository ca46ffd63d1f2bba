"""The norm of query and key heads with the position rotation, forward and
backward, in float64.

Test infrastructure only (see the package docstring).

The paper's model has the Qwen3-1.7B architecture (Section 2): between the QKV
projection and attention every query and key head x of D values is normalised
and turned by its token's position,

    n = x gamma / sqrt(mean(x^2) + eps)
    (a, b) -> (a c - b s, b c + a s)

for the pairs (a, b) = (n_i, n_{i + R/2}) (or (n_2i, n_2i+1), interleaved) of the
first R values, with c and s the cosine and sine of the position's angle for the
pair; the rest of the head stays. The readings: statistics, products and the
rotation in binary32 from the BF16 head, one rounding to BF16; c and s are
binary32 table entries, taken here as given; eps as its binary32 value.

The backward, from the gradient dy of the result: with dn = dy turned back,
r = 1 / sqrt(mean(x^2) + eps), h = x r and g = dn gamma,

    dx = r (g - h mean(g h)),    dgamma = sum over tokens and heads of dn h.

Each function also returns an allowance: how far a binary32 evaluation may be
from the float64 value, u = 2^-24 being half a unit in the last place.
  * r: the sum of squares in any order of the library's depth (8 values a lane,
    then at most 5 additions across lanes) within 14 u, its mean, the root and
    the quotient 5 u more, the root halves what comes before it: 12 u.
  * n: 14 u. A rotated value: two products and a sum of terms |a c| + |b s|:
    16 u of that sum; 2^-19 (32 u) is allowed.
  * dn: 2 u of S = |dy_a c| + |dy_b s|; g: 3 u; h: 13 u; the mean of g h: 31 u of
    the mean of S |gamma| |h|; dx: 64 u = 2^-18 of r (S |gamma| + |h| mean(S |gamma| |h|)).
  * dgamma: terms within 15 u of S |h|, and a sum at most 100 additions deep
    (a lane's tokens and heads, the block, the blocks' partial sums): 2^-17 of sum S |h|.

Parity unpinned by the paper (it prints no values here); pinned in
tests/test_oracle_qk_norm_rope.py by finite differences, by complex
multiplication, by the product of two turned heads depending on the distance of
their positions alone, and by closed forms.
"""

import numpy as np

from . import bf16

FWD_REL, BWD_REL, DGAMMA_REL = 2.0 ** -19, 2.0 ** -18, 2.0 ** -17


def angles(positions, dim, theta):
    """cos and sin [T, dim / 2] of p theta^(-2 i / dim), float64."""
    i = np.arange(dim // 2, dtype=np.float64)
    a = np.asarray(positions, dtype=np.float64)[:, None] * np.float64(theta) ** (-2.0 * i / max(1, dim))
    return np.cos(a), np.sin(a)


def _pairs(dim, interleaved):
    i = np.arange(dim // 2)
    return (2 * i, 2 * i + 1) if interleaved else (i, i + dim // 2)


def rotate(x, cos, sin, interleaved):
    """x [T, H, D] with the first R = 2 cos.shape[1] values of each head turned; and the sum of the magnitudes
    of each result's terms."""
    y, mag = x.copy(), np.abs(x)
    ia, ib = _pairs(2 * cos.shape[1], interleaved)
    a, b = x[..., ia], x[..., ib]
    c, s = cos[:, None, :], sin[:, None, :]
    y[..., ia], y[..., ib] = a * c - b * s, b * c + a * s
    mag[..., ia], mag[..., ib] = np.abs(a * c) + np.abs(b * s), np.abs(b * c) + np.abs(a * s)
    return y, mag


def forward(x, gamma, eps, cos, sin, interleaved=False):
    """(y, allowance) [T, H, D] of heads x, gamma [D] or None, all float64."""
    n = x
    if gamma is not None:
        r = 1.0 / np.sqrt((x * x).mean(axis=-1, keepdims=True) + np.float64(np.float32(eps)))
        n = x * r * gamma
    y, mag = rotate(n, cos, sin, interleaved)
    return y, FWD_REL * mag


def backward(dy, x, gamma, eps, cos, sin, interleaved=False):
    """(dx, allowance, dgamma, allowance) of the gradient dy [T, H, D]; dgamma None without a weight."""
    dn, mag = rotate(dy, cos, -sin, interleaved)
    if gamma is None:
        return dn, BWD_REL * mag, None, None
    r = 1.0 / np.sqrt((x * x).mean(axis=-1, keepdims=True) + np.float64(np.float32(eps)))
    h = x * r
    g = dn * gamma
    dx = r * (g - h * (g * h).mean(axis=-1, keepdims=True))
    sg = mag * np.abs(gamma)
    tol = BWD_REL * r * (sg + np.abs(h) * (sg * np.abs(h)).mean(axis=-1, keepdims=True))
    return dx, tol, (dn * h).sum(axis=(0, 1)), DGAMMA_REL * (mag * np.abs(h)).sum(axis=(0, 1))


def band(ref, tol):
    """BF16 patterns (mid, lo, hi): the rounding of ref, and of the ends of what a binary32 evaluation may give."""
    tol = tol + 2.0 ** -140        # a result below binary32's normal range
    return bf16.from_f64_rne(ref), bf16.from_f64_rne(ref - tol), bf16.from_f64_rne(ref + tol)
