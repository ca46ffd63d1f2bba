"""The quantised backward of the query / key norm on heads and gradients that
do not lie token by token: heads first, padded rows and heads, one gradient for
all heads or all tokens, sequences in padded blocks. Its bytes are those of the
same values laid out densely, which tests/test_gpu_qk_norm_rope.py checks
against the oracle."""

import pytest

from test_gpu_qk_norm_rope import E4, E5, ROW, TENSOR, Case, P  # noqa: F401

pytestmark = pytest.mark.gpu


def heads_first(t):
    return t.transpose(-3, -2).contiguous().transpose(-3, -2)


def padded(t):
    """The same values inside a larger tensor: two tokens, a head and 8 values more in each direction."""
    import torch
    *lead, s, h, d = t.shape
    big = torch.full((*lead, s + 2, h + 1, d + 8), float("nan"), dtype=t.dtype, device=t.device)
    inner = big[..., 1:-1, :-1, :d]
    inner.copy_(t)
    return inner


def one_head(t):
    return t[..., :1, :].expand_as(t)


def one_token(t):
    return t[..., :1, :, :].expand_as(t)


# the whole heads turned by halves whose sequences are groups of 8 tokens, and every other way
FORMS = [(256, 4, 2, 128, 128, False, 2), (256, 5, 1, 64, 64, False, 1), (256, 4, 2, 128, 48, True, 2), (128, 3, 2, 64, 32, False, 1),
         (384, 2, 1, 128, 128, False, 3)]


@pytest.mark.parametrize("T,hq,hk,D,R,inter,batch", FORMS)
@pytest.mark.parametrize("fmt,mode,r", [(E4, ROW, 1), (E5, TENSOR, 0)])
@pytest.mark.parametrize("given", [False, True])
def test_layouts(P, T, hq, hk, D, R, inter, batch, fmt, mode, r, given):  # noqa: F811
    import torch
    if mode == ROW and (hq + 2 * hk) * D % 128:
        hq += 1
    c = Case(P, T + D + hq, T, hq, hk, D, R, inter, positions="given" if given else "rows", batch=batch)
    keep, heads = list(c.g), (c.q, c.k)

    def run():
        return P.qk_norm_rope_bwd_quantize_fp8(*c.g, c.q, c.k, fmt=fmt, mode=mode, rnd=r, want_qT=True, **c.args)

    def same(a, b):
        return all((a[n] is None and b[n] is None) or torch.equal(a[n], b[n]) for n in a)

    want = run()
    for grads in (heads_first, padded):
        c.g = [grads(t) for t in keep]
        assert same(run(), want), grads.__name__
        c.q, c.k = (grads(t) for t in heads)
        assert same(run(), want), "the heads too, " + grads.__name__
        c.q, c.k = heads
    c.g = [heads_first(keep[0]), padded(keep[1]), keep[2]]
    assert same(run(), want), "each its own"
    for spread in (one_head, one_token):
        c.g = [spread(t) for t in keep]
        got = run()
        c.g = [t.contiguous() for t in c.g]
        assert same(got, run()), spread.__name__
