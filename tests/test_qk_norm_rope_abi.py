"""Host-side refusals of the query / key norm calls (no GPU): each invalid
argument returns its documented status before anything is launched."""

import ctypes

import pytest

from test_abi import ERR_ALIGN, ERR_NULL, ERR_SHAPE, ERR_UNSUPPORTED, ERR_WORKSPACE, FAKE, OK, puro  # noqa: F401

BIG = 1 << 40


@pytest.fixture(scope="module")
def call(puro):  # noqa: F811
    L = puro.lib()

    def heads(h):
        return None if h is None else ctypes.byref(puro.Heads(*h))

    def call(which, batch=2, seq=8, hq=4, hk=2, d=64, gq=FAKE, gk=FAKE, eps=1e-6, rope=(FAKE, 16, 64, 0, None), ws=FAKE,
             nb=BIG, fmt=0, mode=0, rnd=0, q8=FAKE, scale=FAKE, qT=None, scaleT=None, dgq=FAKE, dgk=FAKE, **at):
        dense = lambda n: (FAKE, seq * n * d, n * d, d)
        q, k, dq, dk, dv, oq, ok, ov = (at.get(n, dense(hq if n.endswith("q") else hk))
                                        for n in ("q", "k", "dq", "dk", "dv", "oq", "ok", "ov"))
        r = ctypes.byref(puro.RopeArgs(*rope)) if rope else None
        size = (batch, seq, hq, hk, d)
        if which == "fwd":
            return L.puro_qk_norm_rope_fwd(*size, heads(q), heads(k), gq, gk, eps, r, heads(oq), heads(ok), None)
        x = (heads(dq), heads(dk), heads(dv), heads(q), heads(k), gq, gk, eps, r)
        if which == "bwd":
            return L.puro_qk_norm_rope_bwd(*size, *x, heads(oq), heads(ok), heads(ov), dgq, dgk, ws, nb, None)
        return L.puro_qk_norm_rope_bwd_quantize_fp8(*size, *x, fmt, mode, rnd, q8, scale, qT, scaleT, dgq, dgk, ws, nb, None)
    return call


@pytest.mark.parametrize("which", ["fwd", "bwd", "quant"])
def test_refusals_of_all_calls(call, which):
    f = lambda **a: call(which, **a)
    assert f(batch=-1) == f(seq=-1) == f(hq=-1) == f(hk=65536) == ERR_SHAPE
    assert f(batch=1 << 16, seq=1 << 15) == f(batch=1 << 40) == ERR_SHAPE          # 2^31 tokens
    assert f(d=264) == f(d=0) == ERR_SHAPE
    assert f(d=68) == ERR_ALIGN
    for eps in (-1e-6, float("nan"), float("inf")):
        assert f(eps=eps) == ERR_UNSUPPORTED
    assert f(gq=FAKE + 2) == f(gk=FAKE + 8) == ERR_ALIGN
    # the rotation
    assert f(rope=(FAKE, 16, 80, 0, None)) == f(rope=(FAKE, 16, -16, 0, None)) == ERR_SHAPE     # past the head
    assert f(rope=(FAKE, 7, 64, 0, None)) == ERR_SHAPE                                          # 8 positions, 7 entries
    assert f(rope=(FAKE, 0, 64, 0, FAKE)) == f(rope=(FAKE, -1, 64, 0, FAKE)) == f(rope=(FAKE, 1 << 31, 64, 0, FAKE)) == ERR_SHAPE
    assert f(rope=(FAKE, 16, 24, 0, None)) == f(rope=(FAKE + 8, 16, 64, 0, None)) == f(rope=(FAKE, 16, 64, 0, FAKE + 2)) == ERR_ALIGN
    assert f(rope=(None, 16, 64, 0, None)) == ERR_NULL
    assert f(rope=(FAKE, 16, 64, 2, None)) == ERR_UNSUPPORTED
    # the heads
    inputs = ["q", "k"] + (["dq", "dk"] if which != "fwd" else []) + (["dv"] if which == "quant" else [])
    outputs = {"fwd": ["oq", "ok"], "bwd": ["oq", "ok", "ov"], "quant": []}[which]
    for n in inputs + outputs:
        assert f(**{n: None}) == f(**{n: (None, 2048, 256, 64)}) == ERR_NULL, n
        assert f(**{n: (FAKE + 8, 2048, 256, 64)}) == f(**{n: (FAKE, 2048, 260, 64)}) == ERR_ALIGN, n
        assert f(**{n: (FAKE, 2048, -256, 64)}) == f(**{n: (FAKE, 1 << 62, 256, 64)}) == ERR_SHAPE, n
    for n in outputs:
        # heads, tokens or sequences over each other
        for st in ((2048, 256, 56), (2048, 120, 64), (1024, 256, 64), (2048, 256, 0), (0, 256, 64)):
            assert f(**{n: (FAKE, *st)}) == ERR_SHAPE, (n, st)


def test_refusals_of_the_backward(call):
    f = lambda **a: call("bwd", **a)
    assert f(dv=None) == f(ov=None) == ERR_NULL
    assert f(gq=None) == f(gk=None) == ERR_NULL                  # dgamma without gamma
    assert f(dgq=FAKE + 2) == f(ws=FAKE + 8) == ERR_ALIGN
    assert f(ws=None) == ERR_NULL
    assert f(nb=16) == ERR_WORKSPACE


def test_refusals_of_the_quantised_backward(call, puro):  # noqa: F811
    f = lambda **a: call("quant", **a)
    need = puro.lib().puro_qk_norm_rope_bwd_quantize_workspace_size(2, 8, 4, 2, 64)
    assert need > 0 and f(nb=need - 1) == ERR_WORKSPACE
    assert f(ws=None) == f(scale=None) == f(q8=None) == ERR_NULL
    assert f(d=32, rope=None) == f(d=96, rope=None) == f(mode=3, rnd=1) == f(mode=9) == f(fmt=7) == f(rnd=9) == f(mode=1) == ERR_UNSUPPORTED
    assert f(mode=1, rnd=1, qT=FAKE, scaleT=FAKE) == ERR_ALIGN         # 16 rows in column groups
    assert f(seq=4, qT=FAKE) == ERR_ALIGN                              # 8 rows
    assert f(hk=1, hq=1, mode=1, rnd=1) == ERR_ALIGN                   # 192 columns


def test_sizes_and_empty_calls(call, puro):  # noqa: F811
    L = puro.lib()
    assert L.puro_qk_norm_rope_bwd_workspace_size(-1, 8, 64) == 0
    assert L.puro_qk_norm_rope_bwd_workspace_size(1, 8, 60) == 0
    assert 0 < L.puro_qk_norm_rope_bwd_workspace_size(1, 8, 64) <= L.puro_qk_norm_rope_bwd_workspace_size(4, 8192, 64) < 1 << 22
    assert L.puro_qk_norm_rope_bwd_quantize_workspace_size(1, 8, -1, 2, 64) == 0
    # nothing to do: nothing is launched, no pointer is looked at
    none = dict.fromkeys(("q", "k", "dq", "dk", "dv", "oq", "ok", "ov"))
    for size in (dict(batch=0), dict(seq=0)):
        assert call("fwd", **size, **none) == OK
        assert call("bwd", dgq=None, dgk=None, ws=None, nb=0, **size, **none) == OK
        assert call("quant", mode=1, rnd=1, dgq=None, dgk=None, ws=None, nb=0, q8=None, scale=None, **size, **none) == OK


def test_largest_calls(call, puro):  # noqa: F811
    """More tokens than a launch takes are refused, not left to the launch to fail."""
    L = puro.lib()
    far = dict(rope=(FAKE, 16, 64, 0, FAKE))
    for which in ("fwd", "bwd"):
        assert call(which, batch=1, seq=(1 << 25) + 1, **far) == ERR_SHAPE
    assert call("quant", batch=1, seq=(1 << 22) + 16, **far) == ERR_SHAPE
    assert L.puro_qk_norm_rope_bwd_workspace_size(1, 1 << 25, 64) > 0 == L.puro_qk_norm_rope_bwd_workspace_size(1, (1 << 25) + 1, 64)
    assert L.puro_rope_table(FAKE, 1 << 28, 128, 1e4, None) == ERR_SHAPE


def test_table(puro):  # noqa: F811
    f = puro.lib().puro_rope_table
    assert f(FAKE, -1, 64, 1e4, None) == f(FAKE, 1 << 31, 64, 1e4, None) == f(FAKE, 4, 272, 1e4, None) == ERR_SHAPE
    assert f(FAKE, 4, 24, 1e4, None) == f(FAKE + 8, 4, 64, 1e4, None) == ERR_ALIGN
    for theta in (0.0, -1.0, float("inf"), float("nan")):
        assert f(FAKE, 4, 64, theta, None) == ERR_UNSUPPORTED
    assert f(None, 4, 64, 1e4, None) == ERR_NULL
    assert f(None, 0, 64, 1e4, None) == f(None, 4, 0, 1e4, None) == OK
