"""Host-side refusals of the int8 and verification calls (no GPU): each invalid
argument returns its documented status before anything is launched."""

import pytest

from test_abi import ERR_ALIGN, ERR_NULL, ERR_SHAPE, ERR_UNSUPPORTED, ERR_WORKSPACE, FAKE, OK, puro  # noqa: F401

BIG = 1 << 50


def test_quantise(puro):  # noqa: F811
    L = puro.lib()

    def f(x=FAKE, rows=40, cols=64, ld=64, q=FAKE, s=FAKE, qT=FAKE, ldT=48, sT=FAKE, ws=FAKE, nb=BIG):
        return L.puro_quantize_int8(x, rows, cols, ld, q, s, qT, ldT, sT, ws, nb, None)
    assert f(rows=-1) == f(cols=-16) == f(ld=48) == f(ld=1 << 23) == f(ldT=32) == f(ldT=(1 << 22) + 16) == ERR_SHAPE
    assert f(rows=65535 * 128 + 1, ldT=65535 * 129) == ERR_SHAPE
    assert f(cols=56, ld=64) == f(ld=68) == f(x=FAKE + 8) == f(q=FAKE + 8) == f(qT=FAKE + 8) == f(s=FAKE + 2) == ERR_ALIGN
    assert f(sT=FAKE + 2) == f(ldT=56) == f(ws=FAKE + 8) == ERR_ALIGN
    assert f(x=None) == f(s=None) == f(sT=None) == f(ws=None) == f(q=None, qT=None) == ERR_NULL
    need = L.puro_quantize_int8_workspace_size(40, 64)
    assert need > 0 and f(nb=need - 1) == ERR_WORKSPACE
    assert f(rows=0, x=None, q=None, s=None, qT=None, sT=None, ws=None, nb=0) == OK
    assert f(rows=7, cols=0, ld=0, x=None, q=None, s=None, qT=None, sT=None, ws=None, nb=0) == OK
    for bad in ((-1, 16), (0, 16), (4, 0), (1 << 40, 16), (4, 1 << 40)):
        assert L.puro_quantize_int8_workspace_size(*bad) == 0


def test_fused_quantise(puro):  # noqa: F811
    L = puro.lib()

    def norm(x=FAKE, g=FAKE, rows=4, cols=64, ld=64, eps=1e-6, q=FAKE, s=FAKE, r=None):
        return L.puro_rmsnorm_quantize_int8(x, g, rows, cols, ld, eps, q, s, r, None)
    assert norm(rows=-1) == norm(ld=56) == norm(cols=0, ld=0) == norm(ld=1 << 23) == ERR_SHAPE
    assert norm(cols=56) == norm(g=FAKE + 8) == norm(q=FAKE + 4) == norm(s=FAKE + 1) == norm(r=FAKE + 2) == ERR_ALIGN
    assert norm(x=None) == norm(g=None) == norm(q=None) == norm(s=None) == ERR_NULL
    for eps in (-1e-9, float("nan"), float("inf")):
        assert norm(eps=eps) == ERR_UNSUPPORTED
    assert norm(rows=0, x=None, g=None, q=None, s=None) == OK

    def swiglu(x=FAKE, rows=4, cols=64, ld=128, q=FAKE, s=FAKE):
        return L.puro_swiglu_quantize_int8(x, rows, cols, ld, q, s, None)
    assert swiglu(rows=-1) == swiglu(cols=-16) == swiglu(ld=120) == swiglu(cols=1 << 40) == ERR_SHAPE
    assert swiglu(cols=24, ld=128) == swiglu(ld=132) == swiglu(x=FAKE + 8) == swiglu(q=FAKE + 8) == ERR_ALIGN
    assert swiglu(x=None) == swiglu(q=None) == swiglu(s=None) == ERR_NULL
    assert swiglu(rows=0, x=None, q=None, s=None) == swiglu(cols=0, ld=0, x=None, q=None, s=None) == OK


def test_product(puro):  # noqa: F811
    L = puro.lib()

    def f(M=8, N=20, K=64, A=FAKE, lda=64, sa=FAKE, B=FAKE, ldb=64, sb=FAKE, D=FAKE, t=0, ldd=20, acc=0, bias=None, res=None,
          ldr=0, ws=FAKE, nb=BIG):
        return L.puro_int8_gemm(M, N, K, A, lda, sa, B, ldb, sb, D, t, ldd, acc, bias, res, ldr, ws, nb, None)
    assert f(M=-1) == f(N=-1) == f(K=-16) == f(lda=48) == f(ldb=48) == f(ldd=16) == ERR_SHAPE
    assert f(M=(1 << 22) + 1) == f(N=(1 << 22) + 1, ldd=1 << 23) == f(K=131072, lda=131072, ldb=131072) == ERR_SHAPE
    assert f(M=1 << 22, N=(1 << 14) + 4, ldd=1 << 15) == f(lda=(1 << 22) + 16) == ERR_SHAPE
    assert f(K=56) == f(lda=72) == f(ldb=72) == f(ldd=22) == ERR_ALIGN
    for n in ("A", "B", "sa", "sb", "D", "bias", "res"):
        assert f(**{n: FAKE + 8}, **(dict(ldr=20) if n == "res" else {})) == ERR_ALIGN, n
    for n in ("A", "B", "sa", "sb", "D"):
        assert f(**{n: None}) == ERR_NULL, n
    assert f(t=2) == f(acc=1) == f(t=1, bias=FAKE) == f(t=1, res=FAKE, ldr=20) == ERR_UNSUPPORTED
    far = FAKE + (1 << 20)
    assert f(res=far, ldr=16) == f(res=far, ldr=(1 << 22) + 4) == f(res=FAKE, ldr=24) == f(res=FAKE + 32, ldr=20) == ERR_SHAPE
    assert f(res=far, ldr=22) == ERR_ALIGN
    assert f(M=0, A=None, sa=None, D=None) == f(N=0, B=None, sb=None, D=None) == OK
    for bad in ((0, 5, 16), (5, 0, 16), (5, 5, 0), (-1, 5, 16), (1 << 40, 5, 16), (5, 5, 1 << 40)):
        assert L.puro_int8_gemm_workspace_size(*bad) == 0
    # a product that is split over k needs its workspace
    need = L.puro_int8_gemm_workspace_size(512, 512, 65536)
    if need:
        g = lambda **a: f(M=512, N=512, K=65536, lda=65536, ldb=65536, ldd=512, **a)
        assert g(nb=need - 1) == ERR_WORKSPACE and g(ws=None) == ERR_NULL and g(ws=FAKE + 8) == ERR_ALIGN


def test_linear_layer(puro):  # noqa: F811
    import ctypes
    L = puro.lib()
    good = puro.Saved(FAKE, FAKE, FAKE, FAKE)

    def fwd(X=FAKE, W=FAKE, M=13, N=32, K=48, Y=FAKE, saved=good, ws=FAKE, nb=BIG):
        return L.puro_int8_linear_fwd(X, W, M, N, K, Y, ctypes.byref(saved) if saved else None, ws, nb, None)

    def bwd(dY=FAKE, saved=good, M=13, N=32, K=48, dX=FAKE, dW=FAKE, acc=0, ws=FAKE, nb=BIG):
        return L.puro_int8_linear_bwd(dY, ctypes.byref(saved) if saved else None, M, N, K, dX, dW, acc, ws, nb, None)
    for f, size in ((fwd, L.puro_int8_linear_fwd_workspace_size), (bwd, L.puro_int8_linear_bwd_workspace_size)):
        assert f(M=-1) == f(N=-16) == f(K=-16) == f(M=131057) == f(N=131072) == f(K=131072) == ERR_SHAPE
        assert f(N=40) == f(K=40) == f(ws=FAKE + 8) == ERR_ALIGN
        assert f(ws=None) == ERR_NULL and f(nb=size(13, 32, 48) - 1) == ERR_WORKSPACE
        for i in range(4):
            v = [FAKE] * 4
            v[i] = None
            assert f(saved=puro.Saved(*v)) == ERR_NULL, i
            v[i] = FAKE + 8
            assert f(saved=puro.Saved(*v)) == ERR_ALIGN, i
        assert size(-1, 16, 16) == size(4, 8, 16) == size(4, 16, 131072) == 0 < size(1, 16, 16)
    for n in ("X", "W", "Y"):
        assert fwd(**{n: None}) == ERR_NULL and fwd(**{n: FAKE + 8}) == ERR_ALIGN
    assert fwd(M=0, X=None, Y=None) == fwd(N=0, W=None, Y=None) == OK
    assert bwd(dY=None) == bwd(saved=None) == ERR_NULL
    assert bwd(dY=FAKE + 8) == bwd(dX=FAKE + 8) == bwd(dW=FAKE + 8) == ERR_ALIGN
    assert bwd(dX=None, dW=None) == bwd(M=0, dY=None, dX=None, acc=1) == bwd(K=0, dX=None, dW=None) == OK


def test_verification(puro):  # noqa: F811
    L = puro.lib()

    def f(B=3, T=9, rows=6, V=100, kind=0, t=1, p=FAKE, ldp=100, q=FAKE, ldq=100, ids=FAKE, off=FAKE, u=FAKE, us=FAKE, tau=1.0,
          tok=FAKE, acc=FAKE, ws=FAKE, nb=BIG):
        return L.puro_verify_drafts(B, T, rows, V, kind, t, p, ldp, q, ldq, ids, off, u, us, tau, tok, acc, ws, nb, None)
    assert f(B=-1) == f(T=-1) == f(rows=-1) == f(V=0) == f(rows=10) == f(ldp=99) == f(ldq=99) == ERR_SHAPE
    big = (1 << 22) + 1
    assert f(ldp=big) == f(ldq=big) == f(V=(1 << 21) + 1, ldp=1 << 22, ldq=1 << 22) == f(B=(1 << 16) + 1) == ERR_SHAPE
    assert f(T=(1 << 20) + 1) == f(T=1 << 20, V=1 << 16, ldp=1 << 16, ldq=1 << 16) == ERR_SHAPE
    assert f(B=1 << 16, V=1 << 20, ldp=1 << 20, ldq=1 << 20) == ERR_SHAPE
    assert f(kind=2) == f(t=2) == ERR_UNSUPPORTED
    for tau in (-1.0, float("nan"), float("inf"), 1e-7, 2e6):
        assert f(tau=tau) == ERR_UNSUPPORTED
    for n in ("p", "ids", "off", "u", "us", "tok", "acc", "ws"):
        assert f(**{n: None}) == ERR_NULL, n
    for n in ("p", "q", "ids", "off", "u", "us", "tok", "acc"):
        assert f(**{n: FAKE + 2}) == ERR_ALIGN, n
    assert f(ws=FAKE + 8) == f(t=0, p=FAKE + 1) == f(t=0, q=FAKE + 1) == ERR_ALIGN
    need = L.puro_verify_drafts_workspace_size(3, 9, 6, 100)
    assert need > 0 and f(nb=need - 1) == ERR_WORKSPACE
    assert f(B=0, p=None, ids=None, off=None, u=None, us=None, tok=None, acc=None, ws=None, nb=0) == OK
    # outputs over inputs (9 ids and tokens, 4 offsets, 3 counts)
    at = dict(ids=FAKE, off=FAKE + 256, tok=FAKE + 512, acc=FAKE + 768)
    for n, over in (("tok", FAKE + 4), ("tok", FAKE + 256 + 12), ("tok", FAKE + 256 - 32), ("tok", FAKE + 768 + 8), ("acc", FAKE + 32),
                    ("acc", FAKE + 256 + 12), ("acc", FAKE + 256 - 8)):
        assert f(**dict(at, **{n: over})) == ERR_SHAPE, (n, over - FAKE)
    for bad in ((0, 1, 1, 5), (1, 1, 2, 5), (1, 1, 1, 0), (-1, 1, 1, 5), (1, 1 << 20, 1, 1 << 20)):
        assert L.puro_verify_drafts_workspace_size(*bad) == 0



@pytest.mark.parametrize("call", ["gemm", "quant", "verify"])
def test_binding_refuses_other_types_and_devices(puro, call, monkeypatch):  # noqa: F811
    import torch
    monkeypatch.setattr(puro, "_current", lambda: 0)
    x = torch.zeros(4, 32, dtype=torch.bfloat16)
    q, s = torch.zeros(4, 32, dtype=torch.int8), torch.ones(4)
    if call == "gemm":
        for a in ((x, s, q, s), (q, s, q, s), (q.float(), s, q, s)):
            with pytest.raises((TypeError, ValueError)):
                puro.int8_gemm(*a)
    elif call == "quant":
        with pytest.raises(TypeError):
            puro.quantize_int8(x.float())
        with pytest.raises(ValueError):
            puro.quantize_int8(x)                      # (host memory)
    else:
        with pytest.raises(TypeError):
            puro.verify_drafts(x.half(), None, s, s)
        with pytest.raises(ValueError):
            puro.verify_drafts(x, None, torch.zeros(4, dtype=torch.int32), torch.zeros(2, dtype=torch.int32))
