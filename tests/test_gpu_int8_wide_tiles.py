"""int8 product on the wide tiles of large matrices (256 x 256, 256 x 192, 256 x
128): tiles inside the matrix and ragged ones, every kind of output, against the
oracle's exact sums."""

import numpy as np
import pytest

from oracle import int8

from test_gpu_int8 import P, check_product, codes, product, scales  # noqa: F401

from gpu_util import to_dev

pytestmark = pytest.mark.gpu

# by plan: ragged rows and columns; N a multiple of 4 and, the same plan, not
TILES = {(256, 256): [(3086, 3732, 272), (3086, 3730, 272)], (256, 192): [(2318, 3356, 272), (2318, 3355, 272)],
         (256, 128): [(1934, 3732, 2064), (1934, 3729, 2064)]}
SHAPES = [(tile, *s) for tile, shapes in TILES.items() for s in shapes]


def check_plan(P, tile, M, N, K):  # noqa: F811
    p = P.fp8_gemm_plan(M, -(-N // 4) * 4, K)
    assert (p["tile_m"], p["tile_n"], p["splits"]) == (*tile, 1)
    assert M % tile[0] and N % tile[1] and M > 2 * tile[0] and N > 2 * tile[1]


@pytest.mark.parametrize("tile,M,N,K", SHAPES)
@pytest.mark.parametrize("kind", ["bf16", "bias", "residual", "both in place", "fp32", "accumulate"])
def test_wide_tiles(P, tile, M, N, K, kind):  # noqa: F811
    check_plan(P, tile, M, N, K)
    if kind == "bf16":
        product(P, M, N, K, pad=1)
    elif kind == "bias":
        product(P, M, N, K, bias=True, seed=10)
    elif kind == "residual":
        product(P, M, N, K, res="other", pad=1, seed=20)
    elif kind == "both in place":
        product(P, M, N, K, bias=True, res="inplace", seed=30)
    elif kind == "fp32":
        product(P, M, N, K, "fp32", least=-128, pad=1, seed=40)
    else:
        product(P, M, N, K, "fp32", accumulate=True, seed=50)


@pytest.mark.parametrize("tile,M,N,K", SHAPES[::2])
def test_rows_alone_are_the_rows_of_the_whole(P, tile, M, N, K):  # noqa: F811
    """Bit for bit: a row by the kernels of few rows, in a ragged tile and inside the matrix."""
    import torch
    check_plan(P, tile, M, N, K)
    A, B, sa, sb = to_dev(codes(1, M, K)), to_dev(codes(2, N, K)), to_dev(scales(3, M)), to_dev(scales(4, N))
    g = torch.Generator(device="cuda").manual_seed(5)
    bias = torch.randn(N, generator=g, device="cuda").to(torch.bfloat16)
    res = torch.randn(M, N, generator=g, device="cuda").to(torch.bfloat16)
    whole = P.int8_gemm(A, sa, B, sb, bias=bias, residual=res)
    plain = P.int8_gemm(A, sa, B, sb, P.OUT_FP32)
    for rows in (slice(0, 1), slice(300, 316), slice(M - 3, M), slice(200, 261)):
        part = P.int8_gemm(A[rows], sa[rows].clone(), B, sb, bias=bias, residual=res[rows].clone())
        assert torch.equal(part.view(torch.int16), whole[rows].view(torch.int16)), rows
        assert torch.equal(P.int8_gemm(A[rows], sa[rows].clone(), B, sb, P.OUT_FP32), plain[rows]), rows


def test_a_layer_whose_products_are_wide(P):  # noqa: F811
    """The layer's backward on 256-wide tiles: dX (BF16) and dW (FP32, added to) against the products of its own codes."""
    import torch
    M, N, K = 2048, 4096, 8960
    assert P.fp8_gemm_plan(M, K, N)["tile_m"] == P.fp8_gemm_plan(N, K, M)["tile_m"] == 256
    g = torch.Generator(device="cuda").manual_seed(1)
    X, W, dY = (torch.randn(r, c, generator=g, device="cuda").to(torch.bfloat16) for r, c in ((M, K), (N, K), (M, N)))
    _, saved = P.int8_linear_fwd(X, W)
    dW = torch.ones(N, K, device="cuda")
    dX, dW = P.int8_linear_bwd(dY, saved, dW=dW, accumulate_dw=True)
    q = P.quantize_int8(dY, want_qT=True)
    host = lambda t: t.cpu().numpy()                             # noqa: E731
    rows = np.random.default_rng(2).choice(M, 60, replace=False)
    ref, tol = int8.gemm(host(q["q"])[rows], host(q["scale"])[rows], host(saved["wq_t"]), host(saved["w_scale"]))
    check_product(dX[torch.from_numpy(rows).cuda()], ref, tol, "dX")
    rows = np.random.default_rng(3).choice(N, 60, replace=False)
    ref, tol = int8.gemm(host(q["qT"])[rows], host(q["scaleT"])[rows], host(saved["xq_t"]), host(saved["x_scale"]), add=1.0)
    check_product(dW[torch.from_numpy(rows).cuda()], ref, tol, "dW")
