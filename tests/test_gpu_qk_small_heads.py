"""Query / key heads so small that binary32 squares of their values lose bits
or vanish (below 2^-126, 2^-149), where eps is too small to stand over them:
forward and backward against the oracle (oracle/qk_norm_rope.py), the quantised
backward against quantising the BF16 one."""

import numpy as np
import pytest

from oracle import bf16, qk_norm_rope as qk

from gpu_util import bf16_bits, host

pytestmark = pytest.mark.gpu

# sizes of the heads of a call, the last below BF16's normal range (1.2e-38)
SIZES = [1.0, 1e-14, 1e-16, 1e-18, 1e-20, 1e-21, 1e-22, 1e-23, 1e-30, 1e-38, 1e-39, 3.0]


@pytest.fixture(scope="module")
def P():
    from paper_2608_27370_amd import puro
    puro.lib()
    return puro


def f64(bits):
    return bf16.to_f32(np.asarray(bits, dtype=np.uint16)).astype(np.float64)


def dev(bits):
    import torch
    return torch.from_numpy(np.ascontiguousarray(bits).view(np.int16)).cuda().view(torch.bfloat16)


def inside(t, ref, tol, what):
    got = bf16.to_f32(bf16_bits(t.contiguous())).reshape(ref.shape)
    with np.errstate(over="ignore"):
        _, lo, hi = (bf16.to_f32(v) for v in qk.band(ref, tol))
    bad = ~((lo <= got) & (got <= hi))
    assert not bad.any(), "%s: %d of %d outside, first at %s: got %r, between %r and %r" % (
        what, bad.sum(), bad.size, np.argwhere(bad)[0], got[bad][0], lo[bad][0], hi[bad][0])


@pytest.mark.parametrize("eps", [0.0, 1e-40, 1e-33, 1e-6])
@pytest.mark.parametrize("D,R,inter", [(8, 0, False), (64, 64, False), (80, 48, True), (128, 128, False), (256, 64, False)])
def test_small_heads(P, D, R, inter, eps):
    import torch
    g = np.random.default_rng(D)
    T, H = 16, len(SIZES)                                      # (the order changes from token to token)
    size = np.stack([np.roll(SIZES, t) for t in range(T)])[..., None]
    x = bf16.from_f64_rne(g.normal(size=(T, H, D)) * size)
    d = bf16.from_f64_rne(g.normal(size=(T, H, D)) * 1e-3)
    gamma = bf16.from_f64_rne(1 + 0.2 * g.normal(size=D))
    rope = P.rope_table(T, R, 1e4, inter) if R else None
    table = rope.table.cpu().numpy().astype(np.float64) if R else np.zeros((T, 0, 2))
    args = dict(gamma_q=dev(gamma), gamma_k=dev(gamma), rope=rope, eps=eps)
    q, k, dq, dk = dev(x[:, :8]), dev(x[:, 8:]), dev(d[:, :8]), dev(d[:, 8:])
    y = torch.cat(P.qk_norm_rope_fwd(q, k, **args), 1)
    inside(y, *qk.forward(f64(x), f64(gamma), eps, table[..., 0], table[..., 1], inter), "forward")
    out, dgq, dgk = P.qk_norm_rope_bwd(dq, dk, dk, q, k, **args)
    ref, tol, _, _ = qk.backward(f64(d), f64(x), f64(gamma), eps, table[..., 0], table[..., 1], inter)
    inside(out.view(T, -1, D)[:, :H], ref, tol, "backward")
    for got, i in ((dgq, slice(0, 8)), (dgk, slice(8, H))):
        _, _, want, allowed = qk.backward(f64(d)[:, i], f64(x)[:, i], f64(gamma), eps, table[..., 0], table[..., 1], inter)
        assert (np.abs(host(got).astype(np.float64) - want) <= allowed).all()
    if D in (64, 128):
        r = P.qk_norm_rope_bwd_quantize_fp8(dq, dk, dk, q, k, fmt=P.E4M3, mode=P.SCALE_TENSOR, want_qT=True, **args)
        want = P.quantize_fp8(out, P.E4M3, P.SCALE_TENSOR, want_qT=True)
        assert all(torch.equal(r[n], want[n]) for n in ("q", "qT", "scale"))
        torch.testing.assert_close(r["dgamma_q"], dgq, rtol=0, atol=2e-5 * float(dgq.abs().max()))


def test_a_head_of_zeros_without_eps(P):
    """0 / 0, as the formula has it, beside a small head and one of the usual size."""
    import torch
    x = torch.zeros(1, 3, 64, dtype=torch.bfloat16, device="cuda")
    x[0, 1], x[0, 2] = 1e-30, 1.0
    gamma = torch.ones(64, dtype=torch.bfloat16, device="cuda")
    y, _ = P.qk_norm_rope_fwd(x, x[:, :0], gamma_q=gamma, eps=0.0)
    assert torch.isnan(y[0, 0]).all() and (y[0, 1:] == 1).all()
