"""GPU parity of the int8 quantisers, product and linear layer against the
oracle (oracle/int8.py): codes and scales of BF16 tensors bit for bit, those of
the fused norms and SwiGLU within its bands, the product within the roundings of
its binary32 factors and sums (the integer sum itself is exact)."""

import numpy as np
import pytest

from oracle import bf16, int8

from gpu_util import assert_bytes_equal, assert_f32_bits_equal, bf16_bits, host, to_dev, to_dev_bf16

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def P():
    from paper_2608_27370_amd import puro
    puro.lib()
    return puro


def f64(bits):
    return bf16.to_f32(np.asarray(bits, np.uint16)).astype(np.float64)


def activations(seed, R, C):
    g = np.random.default_rng(seed)
    return bf16.from_f64_rne(g.standard_t(3, (R, C)) * np.exp(g.normal(size=(R, 1))) * np.exp(0.5 * g.normal(size=(1, C))))


SHAPES = [(1, 16), (1, 1536), (3, 48), (16, 512), (17, 528), (33, 2048), (128, 2064), (300, 1536), (5, 17920), (2, 65552),
          (257, 4112), (1000, 64), (64, 8960), (4100, 32), (4097, 128), (5003, 112), (385, 4096), (500, 144), (768, 2048),
          (769, 128), (640, 3200), (129, 20480), (129, 20496)]


def check_both(P, x, R, C, dev=None, **kw):
    r = P.quantize_int8(to_dev_bf16(x) if dev is None else dev, want_qT=True, **kw)
    v = f64(x)
    for got, want in ((r["q"], int8.encode_rows(v)), (r["qT"], int8.encode_cols(v))):
        scale = r["scale"] if got is r["q"] else r["scaleT"]
        assert_bytes_equal(host(got), want[0], "%dx%d codes" % (R, C))
        assert_f32_bits_equal(host(scale), want[1], "%dx%d scales" % (R, C))
    return r


@pytest.mark.parametrize("R,C", SHAPES)
def test_codes_and_scales(P, R, C):
    x = activations(R + C, R, C)
    check_both(P, x, R, C)
    one = P.quantize_int8(to_dev_bf16(x))
    assert one["qT"] is None and one["scaleT"] is None
    assert_bytes_equal(host(one["q"]), int8.encode_rows(f64(x))[0])
    other = P.quantize_int8(to_dev_bf16(x), want_q=False, want_qT=True)
    assert other["q"] is None
    assert_bytes_equal(host(other["qT"]), int8.encode_cols(f64(x))[0])


@pytest.mark.parametrize("R,C", [(9000, 64), (2500, 528), (16399, 2064), (701, 48016)])
def test_both_copies_of_long_and_large_tensors(P, R, C):
    g = np.random.default_rng(R)
    x = g.integers(0, 1 << 16, (R, C), dtype=np.uint16)
    x[(x & 0x7F80) > 0x5000] &= 0xCFFF                # (finite, of many magnitudes)
    x[:, : C // 2][: R // 3] = 0
    check_both(P, x, R, C)


def special(R=48, C=64):
    x = activations(9, R, C)
    x[0] = 0
    x[1] = 0x8000
    x[2, 5] = 0x7F80                                  # infinity
    x[3, 6] = 0xFFC1                                  # NaN
    x[4] = np.random.default_rng(1).integers(0, 8, C)           # subnormals
    x[5] = np.random.default_rng(2).integers(0x7F00, 0x7F80, C)      # the largest values
    x[6] = np.random.default_rng(3).integers(0x0080, 0x1800, C)      # about the border where the factor is scaled
    x[:, 8:16][7:] = 0
    x[:7, 8:16] = 0                                   # whole columns of zeros
    return x


def test_special_rows_and_columns(P):
    x = special()
    check_both(P, x, *x.shape)
    check_both(P, np.ascontiguousarray(x.T), *x.T.shape)


@pytest.mark.parametrize("R,C", [(1, 32), (37, 272), (130, 1536)])
def test_strided_input_and_pitched_copy(P, R, C):
    import torch
    wide = activations(R, R, C + 40)
    dev = to_dev_bf16(wide)[:, 8:8 + C]
    pitch = (R + 15) // 16 * 16
    room = torch.full((C, pitch + 32), 77, dtype=torch.int8, device="cuda")
    r = check_both(P, wide[:, 8:8 + C], R, C, dev=dev, out=dict(qT=room[:, :pitch]))
    assert r["qT"].data_ptr() == room.data_ptr()
    assert (host(room)[:, pitch:] == 77).all()                   # what lies behind is left alone


def check_band(q, scale, values, e, what):
    lo, hi, s, tol = int8.band_rows(values, e)
    c = host(q).astype(np.float64)
    bad = ~((lo <= c) & (c <= hi))
    assert not bad.any(), "%s: %d codes outside their band" % (what, bad.sum())
    assert (np.abs(host(scale) - s) <= tol).all(), what
    assert (lo == hi).mean() > 0.99 or values.size < 1000        # (the band leaves almost every code no choice)


@pytest.mark.parametrize("R,C", SHAPES)
def test_rmsnorm(P, R, C):
    x, g = activations(R, R, C), bf16.from_f64_rne(1 + 0.3 * np.random.default_rng(C).normal(size=C))
    x[R // 2] = 0
    r = P.rmsnorm_quantize_int8(to_dev_bf16(x), to_dev_bf16(g), 1e-6, want_rstd=True)
    y, rstd, e = int8.rmsnorm(f64(x), f64(g), np.float64(np.float32(1e-6)))
    check_band(r["q"], r["scale"], y, e, "rmsnorm %dx%d" % (R, C))
    assert (np.abs(host(r["rstd"]) - rstd) <= e * rstd).all()


@pytest.mark.parametrize("R,C", SHAPES)
def test_swiglu(P, R, C):
    gu = activations(C, R, 2 * C)
    gu[R // 2] = 0
    r = P.swiglu_quantize_int8(to_dev_bf16(gu), C)
    h, e = int8.swiglu(f64(gu))
    check_band(r["q"], r["scale"], h, e, "swiglu %dx%d" % (R, C))


def test_fused_strides_and_far_gates(P):
    wide = activations(5, 21, 2 * 96 + 24)
    g = wide[:, 16:16 + 192].copy()
    g[3, :96] = 0xC348                                           # gates of -200: silu is 0
    g[4, :96] = 0xC2A0                                           # and of -80: e^-80
    g[5, :96] = 0x4348
    wide[:, 16:16 + 192] = g
    r = P.swiglu_quantize_int8(to_dev_bf16(wide)[:, 16:16 + 192], 96)
    h, e = int8.swiglu(f64(g))
    h[3] = 0
    check_band(r["q"], r["scale"], h, e, "far gates")
    x = to_dev_bf16(wide)[:, 16:16 + 192]
    gamma = to_dev_bf16(bf16.from_f64_rne(np.ones(192)))
    r = P.rmsnorm_quantize_int8(x, gamma, 0.5)
    y, _, e = int8.rmsnorm(f64(g), np.ones(192), 0.5)
    check_band(r["q"], r["scale"], y, e, "strided norm")


def test_fused_special_rows(P):
    x = activations(6, 5, 128)
    x[1, 3], x[2, 4] = 0x7F80, 0x7FC0
    r = P.rmsnorm_quantize_int8(to_dev_bf16(x), to_dev_bf16(bf16.from_f64_rne(np.ones(128))), 1e-6)
    s = host(r["scale"])
    assert np.isnan(s[2]) and not host(r["q"])[2].any() and np.isfinite(s[[0, 3, 4]]).all()
    assert np.isnan(s[1]) and not host(r["q"])[1].any()          # infinity times a reciprocal root of 0
    r = P.swiglu_quantize_int8(to_dev_bf16(x), 64)
    s = host(r["scale"])
    assert np.isnan(s[1:3]).all() and not host(r["q"])[1:3].any() and np.isfinite(s[[0, 3, 4]]).all()


# ------------------------------------------------------------------- product
def codes(seed, R, C, least=-127):
    return np.random.default_rng(seed).integers(least, 128, (R, C)).astype(np.int8)


def scales(seed, n):
    return np.exp(np.random.default_rng(seed).normal(size=n)).astype(np.float32) * 1e-3


def check_product(D, ref, tol, what):
    if "float32" in str(D.dtype):
        d, lo, hi = host(D).astype(np.float64), ref - tol, ref + tol
        tol32 = 2.0 ** -24 * np.abs(ref)                          # the result's own binary32 rounding
        lo, hi = lo - tol32, hi + tol32
    else:
        d, lo, hi = f64(bf16_bits(D)), f64(bf16.from_f64_rne(ref - tol)), f64(bf16.from_f64_rne(ref + tol))
    bad = ~((lo <= d) & (d <= hi)) & ~(np.isnan(ref) & np.isnan(d))
    assert not bad.any(), "%s: %d of %d off, first at %s: %r, ref %r" % (
        what, bad.sum(), bad.size, tuple(np.argwhere(bad)[0]), d[tuple(np.argwhere(bad)[0])], ref[tuple(np.argwhere(bad)[0])])


def product(P, M, N, K, out="bf16", bias=False, res=None, accumulate=False, least=-127, pad=0, seed=0):
    """One product against the oracle; pad: spare columns of every pitch."""
    import torch
    A, B = codes(seed + 1, M, K + 16 * pad, least), codes(seed + 2, N, K + 16 * pad, least)
    sa, sb = scales(seed + 3, M), scales(seed + 4, N)
    g = np.random.default_rng(seed + 5)
    pitch = (N + 3) // 4 * 4 + 4 * pad
    bb = bf16.from_f64_rne(g.normal(size=N)) if bias else None
    rr = bf16.from_f64_rne(g.normal(size=(M, pitch))) if res else None
    add = g.normal(size=(M, pitch)).astype(np.float32) if accumulate else None
    dA, dB = to_dev(A)[:, :K], to_dev(B)[:, :K]
    kind = torch.float32 if out == "fp32" else torch.bfloat16
    room = torch.full((M, pitch), 7.0, dtype=kind, device="cuda")
    if accumulate:
        room = to_dev(add)
    residual = None
    if res:
        residual = to_dev_bf16(rr)
        if res == "inplace":
            room = residual
        residual = residual[:, :N]
    D = P.int8_gemm(dA, to_dev(sa), dB, to_dev(sb), D=room[:, :N], accumulate=accumulate,
                    bias=to_dev_bf16(bb) if bias else None, residual=residual)
    ref, tol = int8.gemm(A[:, :K], sa, B[:, :K], sb, f64(bb)[None, :] if bias else None, f64(rr)[:, :N] if res else None,
                         add[:, :N].astype(np.float64) if accumulate else None)
    check_product(D, ref, tol, "%dx%dx%d %s" % (M, N, K, out))
    if pitch > N and not res and not accumulate:
        assert (room[:, N:] == 7.0).all().item()                 # columns behind the last are left alone
    return D


PRODUCTS = [(1, 1, 16), (1, 2048, 1536), (2, 30, 64), (5, 1000, 1536), (7, 131, 80), (8, 64, 8960), (15, 77, 1040), (16, 256, 256),
            (17, 272, 2064), (31, 500, 320), (33, 1531, 96), (48, 640, 1536), (63, 129, 144), (64, 64, 64), (65, 1000, 128),
            (77, 1531, 8960), (100, 4100, 512), (128, 128, 128), (129, 257, 400), (200, 2048, 1536), (255, 255, 1008),
            (256, 512, 8192), (300, 700, 272), (513, 1025, 208), (1000, 520, 2048)]


@pytest.mark.parametrize("M,N,K", PRODUCTS)
def test_product(P, M, N, K):
    product(P, M, N, K)
    product(P, M, N, K, "fp32", seed=10)
    product(P, M, N, K, bias=True, res="other", pad=1, seed=20)


@pytest.mark.parametrize("M,N,K", [(1, 30, 64), (9, 129, 1536), (40, 200, 144), (130, 260, 512), (300, 1000, 2048), (64, 64, 16384)])
@pytest.mark.parametrize("kind", ["bias", "inplace", "accumulate", "pitches", "lowest"])
def test_product_kinds(P, M, N, K, kind):
    if kind == "bias":
        product(P, M, N, K, bias=True)
    elif kind == "inplace":
        product(P, M, N, K, res="inplace")
    elif kind == "accumulate":
        product(P, M, N, K, "fp32", accumulate=True)
    elif kind == "pitches":
        product(P, M, N, K, "fp32", pad=3)
    else:
        product(P, M, N, K, least=-128)


@pytest.mark.parametrize("M,N,K", [(130, 257, 512), (300, 999, 208), (513, 1027, 64), (70, 131, 16)])
def test_columns_past_the_last_vector_of_four(P, M, N, K):
    product(P, M, N, K, bias=True, res="other")
    product(P, M, N, K, res="inplace")
    product(P, M, N, K, "fp32", accumulate=True)
    product(P, M, N, K, "fp32", pad=1)


# rows and columns of the streaming kernels: whole and ragged groups of 16 rows, the longest reductions that stay in LDS
@pytest.mark.parametrize("M", [1, 5, 16, 17, 32, 33, 49, 64])
@pytest.mark.parametrize("N,K", [(32768, 144), (33000, 2048), (32771, 1536), (40000, 16), (9001, 2032), (20000, 2064)])
def test_few_rows_of_wide_products(P, M, N, K):
    product(P, M, N, K, "fp32")
    product(P, M, N, K, bias=True, res="inplace", seed=30)


@pytest.mark.parametrize("M,N", [(1, 16), (20, 24), (150, 300)])
def test_longest_sums_are_exact(P, M, N):
    """Codes of -128 over the longest reduction: sums just below 2^31."""
    import torch
    K = 131056
    A, B = (torch.full((n, K), -128, dtype=torch.int8, device="cuda") for n in (M, N))
    one = torch.ones(max(M, N), device="cuda")
    D = P.int8_gemm(A, one[:M], B, one[:N], P.OUT_FP32)
    assert (D == float(np.float32(128 * 128 * K))).all().item()
    B[:, ::2] = 127
    D = P.int8_gemm(A, one[:M], B, one[:N], P.OUT_FP32)
    assert (D == float(np.float32(128 * 64 * K - 128 * 127 // 2 * K))).all().item()


def test_empty_sums_and_nan_scales(P):
    import torch
    s = torch.ones(40, device="cuda")
    z = torch.zeros(40, 0, dtype=torch.int8, device="cuda")
    bias = to_dev_bf16(bf16.from_f64_rne(np.arange(24.0)))
    D = P.int8_gemm(z[:8], s[:8], z[:24], s[:24], bias=bias)
    assert torch.equal(D, bias.expand(8, 24))
    assert P.int8_gemm(z[:0], s[:0], z[:24], s[:24]).shape == (0, 24)
    wide = torch.zeros(300, 0, dtype=torch.int8, device="cuda")
    D = P.int8_gemm(wide, torch.ones(300, device="cuda"), wide, torch.ones(300, device="cuda"), P.OUT_FP32)
    assert D.shape == (300, 300) and not D.any().item()
    empty = P.quantize_int8(torch.empty(0, 32, dtype=torch.bfloat16, device="cuda"), want_qT=True)
    assert empty["qT"].shape == (32, 0) and (empty["scaleT"] == 1).all().item()
    x = activations(3, 8, 64)
    x[2, 1], x[5, 60] = 0x7F80, 0x7FC0
    q = P.quantize_int8(to_dev_bf16(x))
    w = P.quantize_int8(to_dev_bf16(activations(4, 24, 64)))
    bad = torch.isnan(P.int8_gemm(q["q"], q["scale"], w["q"], w["scale"])).any(dim=1)
    assert bad.tolist() == [False, False, True, False, False, True, False, False]


def test_refusals_of_the_binding(P):
    import torch
    q, s = torch.zeros(8, 32, dtype=torch.int8, device="cuda"), torch.ones(8, device="cuda")
    for a, kw in (((q, s, q[:, :16], s), {}), ((q, s[:7], q, s), {}), ((q, s, q, s.double()), {}), ((q.t(), s, q, s), {}),
                  ((q, s, q, s), dict(D=torch.zeros(8, 9, device="cuda"))), ((q, s, q, s), dict(D=torch.zeros(8, 8).cuda().half())),
                  ((q, s, q, s), dict(residual=torch.zeros(8, 7, device="cuda", dtype=torch.bfloat16))),
                  ((q, s, q, s), dict(bias=torch.zeros(7, device="cuda", dtype=torch.bfloat16)))):
        with pytest.raises((TypeError, ValueError)):
            P.int8_gemm(*a, **kw)
    with pytest.raises(P.PuroError):
        P.int8_gemm(q, s, q, s, accumulate=True)
    x = torch.zeros(8, 32, dtype=torch.bfloat16, device="cuda")
    for kw in (dict(want_qT=True, out=dict(qT=torch.zeros(32, 8, dtype=torch.int8, device="cuda"))),
               dict(out=dict(q=torch.zeros(8, 32, device="cuda"))), dict(out=dict(scale=torch.zeros(9, device="cuda")))):
        with pytest.raises((TypeError, ValueError)):
            P.quantize_int8(x, **kw)
    with pytest.raises(ValueError):
        P.swiglu_quantize_int8(x, 32)
    with pytest.raises(ValueError):
        P.rmsnorm_quantize_int8(x, x[0, :16], 1e-6)


# -------------------------------------------------------------- linear layer
@pytest.mark.parametrize("M,N,K", [(1, 32, 48), (13, 64, 32), (100, 208, 336), (333, 512, 272)])
def test_linear_and_its_gradients(P, M, N, K):
    """Y, dX and dW against the oracle's products of its own codes; against the exact gradients of sum(dY * X W^T), by the
    formula and by central differences (of a bilinear function: exact up to rounding), within half a step of every code."""
    import torch
    x, w, dy = activations(1, M, K), bf16.from_f64_rne(np.random.default_rng(2).normal(size=(N, K)) * 0.05), activations(3, M, N)
    X, W = (to_dev_bf16(v).requires_grad_() for v in (x, w))
    X3 = X.view(1, M, K)
    Y = P.int8_linear(X3, W)
    assert Y.shape == (1, M, N)
    (xq, xs), (wq, ws), (dq, ds) = (int8.encode_rows(f64(v)) for v in (x, w, dy))
    (xt, xts), (wt, wts), (dt, dts) = (int8.encode_cols(f64(v)) for v in (x, w, dy))
    check_product(Y.detach()[0], *int8.gemm(xq, xs, wq, ws), "Y")
    Y.backward(to_dev_bf16(dy).view(1, M, N))
    check_product(X.grad, *int8.gemm(dq, ds, wt[:, :N], wts), "dX")
    ref, tol = int8.gemm(dt, dts, xt, xts)
    # (W's gradient is handed over in W's type: dW's binary32 rounding, then BF16's)
    check_product(W.grad, ref, tol + 2.0 ** -24 * np.abs(ref), "dW")

    xv, wv, dv = f64(x), f64(w), f64(dy)
    f = lambda a, b: float((dv * (a @ b.T)).sum())                # noqa: E731
    half = 0.5 + 127 * 2.0 ** -22          # (the factor's and the scale's binary32 roundings: 2^-24 each of up to 127 steps)
    for name, grad, exact, p, sp, q, sq in (("dX", X.grad, dv @ wv, dv, ds[:, None], wv, wts[None, :]),
                                            ("dW", W.grad, dv.T @ xv, dv.T, dts[:, None], xv, xts[None, :])):
        # |p' q' - p q| <= |p'| |q' - q| + |p' - p| |q|, each code half a step off; BF16's rounding of the result
        bound = (np.abs(p) + half * sp) @ np.broadcast_to(half * sq, q.shape) + (half * sp * np.ones_like(p)) @ np.abs(q)
        got = f64(bf16_bits(grad))
        assert (np.abs(got - exact) <= bound * (1 + 2.0 ** -20) + (2.0 ** -8 + 2.0 ** -20) * np.abs(got) + 1e-30).all(), name
    h = 0.5
    for m, k in ((0, 0), (M - 1, K - 1)):
        e = np.zeros_like(xv)
        e[m, k] = h
        diff = (f(xv + e, wv) - f(xv - e, wv)) / (2 * h)
        assert abs(diff - (dv @ wv)[m, k]) <= 1e-9 * (1 + np.abs(dv).sum() * np.abs(wv).max() * np.abs(xv).max())


def test_linear_accumulates_into_main_grad(P):
    import torch
    M, N, K = 40, 64, 48
    X, W = (to_dev_bf16(activations(s, r, K)).requires_grad_() for s, r in ((1, M), (2, N)))
    W.main_grad = torch.zeros(N, K, device="cuda")
    dY = to_dev_bf16(activations(3, M, N))
    for _ in range(2):
        P.int8_linear(X, W).backward(dY)
    assert W.grad is None
    _, saved = P.int8_linear_fwd(X.detach(), W.detach())
    _, dW = P.int8_linear_bwd(dY, saved, want_dx=False)
    assert torch.equal(W.main_grad, dW + dW)
    Y = P.int8_linear(X.detach(), W)
    assert Y.requires_grad
    P.int8_linear(X, W.detach()).sum().backward()                 # an expanded gradient; dX alone
    with torch.no_grad():
        assert torch.equal(P.int8_linear(X, W).view(torch.int16), Y.detach().view(torch.int16))
    # rows that do not begin at 16 bytes, of the input and of the gradient
    room = torch.zeros(M * K + 4, dtype=torch.bfloat16, device="cuda")
    odd = room[4:].view(M, K)
    odd.copy_(X.detach())
    odd = odd.requires_grad_()
    Z = P.int8_linear(odd, W)
    grad = torch.zeros(M * N + 1, dtype=torch.bfloat16, device="cuda")[1:].view(M, N)
    Z.backward(grad.copy_(dY))
    X.grad = None
    P.int8_linear(X, W).backward(dY)
    assert torch.equal(odd.grad.view(torch.int16), X.grad.view(torch.int16))
    with pytest.raises(TypeError):
        P.int8_linear(X.float(), W)


@pytest.mark.parametrize("M,N,K", [(0, 32, 48), (1, 16, 16), (21, 48, 64)])
def test_linear_calls_are_the_calls_they_are_made_of(P, M, N, K):
    """(and without what one does not want, and no tokens at all)"""
    import torch
    X, W, dY = (to_dev_bf16(activations(s, r, c)) for s, r, c in ((1, M, K), (2, N, K), (3, M, N)))
    Y, saved = P.int8_linear_fwd(X, W)
    w = P.quantize_int8(W, want_qT=True)
    if M:
        x = P.quantize_int8(X, want_qT=True)
        assert torch.equal(Y.view(torch.int16), P.int8_gemm(x["q"], x["scale"], w["q"], w["scale"]).view(torch.int16))
        for got, want in ((saved["xq_t"], x["qT"]), (saved["x_scale"], x["scaleT"]), (saved["wq_t"], w["qT"]), (saved["w_scale"], w["scaleT"])):
            assert torch.equal(got, want)
    only, none = P.int8_linear_fwd(X, W, want_saved=False)
    assert none is None and torch.equal(only.view(torch.int16), Y.view(torch.int16))
    dX, dW = P.int8_linear_bwd(dY, saved)
    assert dX.shape == (M, K) and dW.shape == (N, K)
    if M == 0:
        assert not dW.any().item()
    kept = torch.full((N, K), 3.0, device="cuda")
    none, same = P.int8_linear_bwd(dY, saved, want_dx=False, dW=kept, accumulate_dw=True)
    assert none is None and same is kept and torch.equal(kept, 3.0 + dW)
    alone, none = P.int8_linear_bwd(dY, saved, want_dw=False)
    assert none is None and torch.equal(alone.view(torch.int16), dX.view(torch.int16))


# ------------------------------------------------- together, streams, graphs
def test_decoder_mlp_in_a_graph_with_eager_work_between(P):
    """norm -> gate/up -> SwiGLU -> down into the residual stream, as one decoding step of an int8 model: replayed on
    other inputs, each replay equal to the eager calls, and both equal to the oracle's chain on its own codes."""
    import torch
    M, K, F = 3, 256, 512
    gamma = to_dev_bf16(bf16.from_f64_rne(1 + 0.1 * np.random.default_rng(0).normal(size=K)))
    up, down = (P.quantize_int8(to_dev_bf16(activations(s, n, k))) for s, n, k in ((1, 2 * F, K), (2, K, F)))
    x = to_dev_bf16(activations(3, M, K))
    out = torch.empty_like(x)

    def step():
        a = P.rmsnorm_quantize_int8(x, gamma, 1e-6)
        gu = P.int8_gemm(a["q"], a["scale"], up["q"], up["scale"])
        h = P.swiglu_quantize_int8(gu, F)
        return a, gu, h, P.int8_gemm(h["q"], h["scale"], down["q"], down["scale"], D=out, residual=x)
    a, gu, h, y = step()
    y64, _, e = int8.rmsnorm(f64(bf16_bits(x)), f64(bf16_bits(gamma)), np.float64(np.float32(1e-6)))
    check_band(a["q"], a["scale"], y64, e, "norm")
    check_product(gu, *int8.gemm(host(a["q"]), host(a["scale"]), host(up["q"]), host(up["scale"])), "gate/up")
    h64, e = int8.swiglu(f64(bf16_bits(gu)))
    check_band(h["q"], h["scale"], h64, e, "swiglu")
    check_product(y, *int8.gemm(host(h["q"]), host(h["scale"]), host(down["q"]), host(down["scale"]),
                                residual=f64(bf16_bits(x))), "down")
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step()
    torch.cuda.current_stream().wait_stream(side)
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        step()
    for r in range(4):
        x.copy_(to_dev_bf16(activations(10 + r, M, K)))
        want = step()[3].clone()
        out.zero_()
        g.replay()
        torch.cuda.synchronize()
        assert torch.equal(out.view(torch.int16), want.view(torch.int16)), r
    del g


def test_two_streams_with_their_own_tensors(P):
    import torch
    X = [to_dev_bf16(activations(s, 777, 512)) for s in (1, 2)]
    W = P.quantize_int8(to_dev_bf16(activations(3, 512, 512)))

    def call(x):
        q = P.quantize_int8(x, want_qT=True)
        return P.int8_gemm(q["q"], q["scale"], W["q"], W["scale"]), P.int8_gemm(q["qT"], q["scaleT"], q["qT"], q["scaleT"], P.OUT_FP32)
    want = [call(x) for x in X]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in X]
    got = [[] for _ in X]
    for _ in range(5):
        for s, x, g in zip(streams, X, got):
            with torch.cuda.stream(s):
                g.append(call(x))
    torch.cuda.synchronize()
    for g, w in zip(got, want):
        for y, z in g:
            assert torch.equal(y.view(torch.int16), w[0].view(torch.int16)) and torch.equal(z, w[1])
