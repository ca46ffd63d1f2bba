"""int8 product: sum, scales and what follows are rounded one after the other,
whichever kernel and whichever part of a tile an output comes from. Every output is
1 x (1 + x) x (1 + 2^-12) - 1 here, x = 2^-12 + 2^-18 + 2^-19 - 2^-23: the product
is T' = 1 + T - 2^-24 + 2^-30 + 2^-31 - 2^-35 with T = 2^-11 + 2^-18 + 2^-19, rounded
to binary32 1 + T, from which 1 (a bias, a residual, what D held) leaves T, in BF16
a tie that goes to the even neighbour above, 2^-11 (1 + 2^-6). Fused into the
subtraction the product leaves less than T: another binary32 number, and in BF16 the
neighbour below, 2^-11 (1 + 2^-7)."""

import numpy as np
import pytest

pytestmark = pytest.mark.gpu

X = 2.0 ** -12 + 2.0 ** -18 + 2.0 ** -19 - 2.0 ** -23
T = 2.0 ** -11 + 2.0 ** -18 + 2.0 ** -19
BF16 = 2.0 ** -11 * (1 + 2.0 ** -6)


def test_the_values_are_what_the_docstring_says():
    a, b = np.float32(1 + X), np.float32(1 + 2.0 ** -12)
    assert float(a) == 1 + X and float(b) == 1 + 2.0 ** -12
    assert float(a) * float(b) < 1 + T                           # (exact in binary64: 36 bits)
    assert np.float32(a * b) == np.float32(1 + T) and np.float32(1 + T) - np.float32(1) == np.float32(T)


@pytest.fixture(scope="module")
def P():
    from paper_2608_27370_amd import puro
    puro.lib()
    return puro


# (rows, columns, k) with the plan of each: none (a kernel of few rows), 64, 128 and 256 wide tiles inside the
# matrix and at its edges, ranges of k summed afterwards
SHAPES = [(1, 2048, 64, None), (16, 40000, 64, None), (16, 4099, 64, None), (50, 300, 64, None), (77, 2060, 1552, (64, 64, 1)),
          (77, 1531, 8960, (64, 64, 5)), (256, 512, 8192, None), (590, 636, 272, (128, 128, 1)), (1934, 3732, 2064, (256, 128, 1)),
          (1934, 3731, 2064, (256, 128, 1)), (2318, 3356, 272, (256, 192, 1)), (2318, 3355, 272, (256, 192, 1)),
          (3086, 3732, 272, (256, 256, 1)), (3086, 3729, 272, (256, 256, 1))]


@pytest.mark.parametrize("M,N,K,plan", SHAPES)
@pytest.mark.parametrize("kind", ["bias", "residual", "in place", "accumulate"])
def test_products_are_rounded_before_what_follows(P, M, N, K, plan, kind):
    import torch
    if plan:
        p = P.fp8_gemm_plan(M, -(-N // 4) * 4, K)
        assert (p["tile_m"], p["tile_n"], p["splits"]) == plan
    A, B = (torch.zeros(n, K, dtype=torch.int8, device="cuda") for n in (M, N))
    A[:, K - 1] = B[:, K - 1] = 1
    sa, sb = torch.full((M,), 1 + X, device="cuda"), torch.full((N,), 1 + 2.0 ** -12, device="cuda")
    pitch = -(-N // 8) * 8
    f32 = kind == "accumulate"
    D = torch.full((M, pitch), -1.0, dtype=torch.float32 if f32 else torch.bfloat16, device="cuda")[:, :N]
    minus = torch.full((M, pitch), -1.0, dtype=torch.bfloat16, device="cuda")[:, :N]
    P.int8_gemm(A, sa, B, sb, D=D, accumulate=f32, bias=minus[0] if kind == "bias" else None,
                residual=D if kind == "in place" else minus if kind == "residual" else None)
    off = D != (T if f32 else BF16)
    assert not off.any().item(), "%d of %d, first at %s: %r" % (off.sum().item(), M * N, off.nonzero()[0].tolist(), D[off][0].item())
