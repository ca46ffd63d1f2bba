"""GPU parity of the query / key norm with rotation (puro_qk_norm_rope_fwd,
puro_qk_norm_rope_bwd, puro_qk_norm_rope_bwd_quantize_fp8, puro_rope_table)
against the oracle (oracle/qk_norm_rope.py): every BF16 result between the
roundings of the ends of the oracle's allowance, dgamma within its allowance,
quantised results by tests/band_check.py."""

import numpy as np
import pytest

from oracle import bf16, fp8, qk_norm_rope as qk

import band_check
from gpu_util import bf16_bits, host, to_dev

pytestmark = pytest.mark.gpu

E4, E5 = 0, 1
TENSOR, ROW, COL, KMAJOR = 0, 1, 2, 0x100
EPS = 1e-6


@pytest.fixture(scope="module")
def P():
    from paper_2608_27370_amd import puro
    puro.lib()
    return puro


def f64(bits):
    return bf16.to_f32(np.asarray(bits, dtype=np.uint16)).astype(np.float64)


def rnd(g, shape, std=1.0):
    return bf16.from_f64_rne(g.normal(size=shape) * std)


def dev(bits, batch=None):
    """BF16 patterns to the device; batch: [T, ..] as [batch, T / batch, ..]."""
    import torch
    t = torch.from_numpy(np.ascontiguousarray(bits).view(np.int16)).cuda().view(torch.bfloat16)
    return t if batch is None else t.unflatten(0, (batch, -1))


class Case:
    """Inputs of one call, on the host (BF16 patterns, [T, H, D]) and as the kernels take them."""

    def __init__(self, P, seed, T, hq, hk, D, R, inter=False, norm="both", positions="rows", batch=1, theta=1e4):
        import torch
        g = np.random.default_rng(seed)
        self.T, self.hq, self.hk, self.D, self.R, self.inter, self.batch = T, hq, hk, D, R, inter, batch
        C = (hq + 2 * hk) * D
        self.qkv = rnd(g, (T, C), np.exp(g.normal(size=C)))
        x = self.qkv.reshape(T, hq + 2 * hk, D)
        self.x = x[:, :hq], x[:, hq:hq + hk]
        gamma = [bf16.from_f64_rne(1 + 0.2 * g.normal(size=D)) for _ in range(2)]
        self.gamma = [gamma[i] if norm in ("both", ("q", "k")[i]) else None for i in range(2)]
        self.d = [rnd(g, (T, h, D), 1e-2) for h in (hq, hk, hk)]
        S = T // batch
        length = max(1, 2 * T)
        self.pos = np.tile(np.arange(S), batch)
        self.p_dev = None
        if positions == "given":
            self.pos = g.integers(0, length, T)
            self.p_dev = torch.from_numpy(self.pos.astype(np.int32)).cuda()
        # the table as the library makes it, checked by itself below
        self.rope = P.rope_table(length, R, theta, inter) if R else None
        if R:
            table = self.rope.table.cpu().numpy().astype(np.float64)
            self.cos, self.sin = table[self.pos, :, 0], table[self.pos, :, 1]
        else:
            self.cos = self.sin = np.zeros((T, 0))
        B = batch if batch > 1 else None
        h = dev(self.qkv, B).unflatten(-1, (hq + 2 * hk, D))
        self.q, self.k = h[..., :hq, :], h[..., hq:hq + hk, :]
        self.args = dict(gamma_q=dev(gamma[0]) if self.gamma[0] is not None else None,
                         gamma_k=dev(gamma[1]) if self.gamma[1] is not None else None, rope=self.rope,
                         positions=self.p_dev, eps=EPS)
        self.g = [dev(v, B) for v in self.d]

    def forward(self, i):
        gm = f64(self.gamma[i]) if self.gamma[i] is not None else None
        return qk.forward(f64(self.x[i]), gm, EPS, self.cos, self.sin, self.inter)

    def backward(self, i):
        gm = f64(self.gamma[i]) if self.gamma[i] is not None else None
        return qk.backward(f64(self.d[i]), f64(self.x[i]), gm, EPS, self.cos, self.sin, self.inter)


def check_band(t, ref, tol, what):
    got = bf16.to_f32(bf16_bits(t.contiguous())).reshape(ref.shape)
    _, lo, hi = (bf16.to_f32(v) for v in qk.band(ref, tol))
    bad = ~((lo <= got) & (got <= hi))
    assert not bad.any(), "%s: %d of %d outside, first at %s: got %r, between %r and %r" % (
        what, bad.sum(), bad.size, np.argwhere(bad)[0], got[bad][0], lo[bad][0], hi[bad][0])


def check_forward(P, c, **out):
    q, k = P.qk_norm_rope_fwd(c.q, c.k, **c.args, **out)
    for i, t in enumerate((q, k)):
        check_band(t, *c.forward(i), "forward %s" % "qk"[i])
    return q, k


def check_dgamma(got, c, i, what):
    if c.gamma[i] is None:
        assert got is None
        return
    _, _, ref, tol = c.backward(i)
    err = np.abs(host(got).astype(np.float64) - ref)
    assert (err <= tol + 1e-30).all(), (what, float((err / (tol + 1e-30)).max()))


def check_backward(P, c, dv=True):
    out, dgq, dgk = P.qk_norm_rope_bwd(c.g[0], c.g[1], c.g[2] if dv else None, c.q, c.k, **c.args)
    heads = out.view(c.T, -1, c.D)
    for i, at in ((0, slice(0, c.hq)), (1, slice(c.hq, c.hq + c.hk))):
        check_band(heads[:, at], *c.backward(i)[:2], "backward %s" % "qk"[i])
    if dv:
        assert (bf16_bits(heads[:, c.hq + c.hk:].contiguous()) == c.d[2]).all()
    else:
        assert heads.shape[1] == c.hq + c.hk
    check_dgamma(dgq, c, 0, "dgamma_q")
    check_dgamma(dgk, c, 1, "dgamma_k")
    return out


# ---------------------------------------------------------------------- table
@pytest.mark.parametrize("length,dim,theta", [(1, 16, 1e4), (777, 48, 1e6), (70000, 128, 1e6), (3, 256, 500000.0)])
def test_table(P, length, dim, theta):
    """Double-precision angles (their error, some 2^-52 of an angle up to 7e4, is below 2^-35) rounded once."""
    r = P.rope_table(length, dim, theta)
    assert r.dim == dim and r.table.shape == (length, dim // 2, 2)
    cos, sin = qk.angles(np.arange(length), dim, theta)
    got = host(r.table).astype(np.float64)
    assert np.abs(got[..., 0] - cos).max() <= 2.0 ** -25 + 2.0 ** -34
    assert np.abs(got[..., 1] - sin).max() <= 2.0 ** -25 + 2.0 ** -34


# --------------------------------------------------------- forward and backward
SHAPES = [
    # T, hq, hk, D, R
    (1, 1, 1, 8, 0), (5, 3, 1, 16, 16), (9, 2, 2, 24, 16), (33, 4, 2, 32, 32), (130, 9, 3, 64, 32),
    (65, 12, 2, 128, 128), (17, 16, 8, 128, 128), (40, 10, 5, 80, 64), (31, 6, 6, 96, 96), (22, 5, 1, 128, 48),
    (19, 4, 4, 192, 96), (12, 3, 1, 256, 256), (7, 40, 3, 64, 64), (3, 1, 9, 128, 0),
]


@pytest.mark.parametrize("T,hq,hk,D,R", SHAPES)
@pytest.mark.parametrize("inter", [False, True])
def test_shapes(P, T, hq, hk, D, R, inter):
    c = Case(P, T * 7 + D, T, hq, hk, D, R, inter, positions="given" if T % 2 else "rows")
    check_forward(P, c)
    check_backward(P, c)


@pytest.mark.parametrize("norm", ["none", "q", "k"])
@pytest.mark.parametrize("R", [0, 32, 128])
def test_norm_of_one_kind_or_none(P, norm, R):
    c = Case(P, 11, 21, 4, 2, 128, R, norm=norm)
    check_forward(P, c)
    check_backward(P, c, dv=norm != "q")


def test_many_tokens_per_wave(P):
    """More tokens than the backward has waves at once, the forward unsplit."""
    c = Case(P, 12, 9001, 2, 1, 64, 64, positions="given")
    check_forward(P, c)
    check_backward(P, c)


@pytest.mark.parametrize("hq,hk", [(3, 0), (0, 2)])
def test_one_kind_of_heads(P, hq, hk):
    c = Case(P, 13, 10, hq, hk, 64, 64)
    check_forward(P, c)
    check_backward(P, c)


@pytest.mark.parametrize("batch", [1, 3])
def test_layouts(P, batch):
    """Heads first, padded rows and heads, a gradient expanded over its heads; positions start again per sequence."""
    import torch
    c = Case(P, 14, 24, 4, 2, 64, 64, batch=batch)
    S = 24 // batch
    plain = check_forward(P, c)
    lead = (batch,) if batch > 1 else ()
    first = [torch.empty(*lead, h, S, 64, dtype=torch.bfloat16, device="cuda").transpose(-3, -2) for h in (4, 2)]
    check_forward(P, c, q_out=first[0], k_out=first[1])
    pad = [torch.full((*lead, S + 2, h, 72), 7.0, dtype=torch.bfloat16, device="cuda") for h in (4, 2)]
    inner = [p[..., 1:-1, :, :64] for p in pad]
    check_forward(P, c, q_out=inner[0], k_out=inner[1])
    for p, i, want in zip(pad, inner, plain):
        assert torch.equal(i, want)
        i.fill_(7.0)
        assert (p == 7.0).all()                                # nothing else was written
    want = bf16_bits(check_backward(P, c))
    # gradients heads first
    keep = list(c.g)
    c.g = [v.transpose(-3, -2).contiguous().transpose(-3, -2) for v in keep]
    assert not c.g[0].is_contiguous()
    assert (bf16_bits(check_backward(P, c)) == want).all()
    # one gradient for all heads of a kind, and one for all tokens
    c.g = [keep[0][..., :1, :].expand_as(keep[0]), keep[1][..., :1, :, :].expand_as(keep[1]), keep[2]]
    c.d = [bf16_bits(v.contiguous()).reshape(24, -1, 64) for v in c.g]
    check_backward(P, c)


def test_in_place(P):
    import torch
    c = Case(P, 15, 19, 4, 2, 128, 128)
    q, k = check_forward(P, c)
    want = bf16_bits(check_backward(P, c))
    # the gradients of q and k over the incoming ones, through the C entry
    dq, dk = c.g[0].clone(), c.g[1].clone()
    H = lambda t: P._heads(t, "t", t.shape, 0)
    L = P.lib()
    assert L.puro_qk_norm_rope_bwd(1, 19, 4, 2, 128, H(dq), H(dk), None, H(c.q), H(c.k), c.args["gamma_q"].data_ptr(),
                                   c.args["gamma_k"].data_ptr(), EPS, P._rope_args(c.rope, None, 19, 0), H(dq), H(dk), None,
                                   None, None, None, 0, P._stream()) == 0
    assert (np.concatenate((bf16_bits(dq), bf16_bits(dk)), 1).reshape(19, -1) == want.reshape(19, -1)[:, :6 * 128]).all()
    P.qk_norm_rope_fwd(c.q, c.k, q_out=c.q, k_out=c.k, **c.args)
    assert torch.equal(c.q, q) and torch.equal(c.k, k)


def test_empty(P):
    import torch
    c = Case(P, 16, 0, 4, 2, 64, 64)
    q, k = P.qk_norm_rope_fwd(c.q, c.k, **c.args)
    assert q.shape == (0, 4, 64) and k.shape == (0, 2, 64)
    out, dgq, dgk = P.qk_norm_rope_bwd(c.g[0], c.g[1], c.g[2], c.q, c.k, **c.args)
    assert out.shape == (0, 8 * 64) and (dgq == 0).all() and (dgk == 0).all()
    for mode, r in ((TENSOR, 0), (ROW, 1)):
        r = P.qk_norm_rope_bwd_quantize_fp8(c.g[0], c.g[1], c.g[2], c.q, c.k, mode=mode, rnd=r, want_qT=True, **c.args)
        assert r["q"].shape == (0, 512) and (r["dgamma_q"] == 0).all() and (r["dgamma_k"] == 0).all()
        assert mode == ROW or r["scale"].item() == 1.0
    torch.cuda.synchronize()


def test_special_values(P):
    """A head of zeros, an infinity (its head NaN or infinite, no other), the largest values whose squares fit."""
    c = Case(P, 17, 6, 2, 1, 64, 32)
    x = c.qkv.reshape(6, -1, 64)
    x[1, 0] = 0
    x[2, 1, 40] = 0x7F80
    x[3, 0] = bf16.from_f64_rne(np.full(64, 1e18))
    x[4, 0] = bf16.from_f64_rne(np.full(64, 1e-30))
    h = dev(c.qkv).unflatten(-1, (4, 64))
    c.q, c.k = h[:, :2], h[:, 2:3]
    q, k = P.qk_norm_rope_fwd(c.q, c.k, **c.args)
    with np.errstate(invalid="ignore"):
        ref, tol = c.forward(0)
    live = np.ones((6, 2), bool)
    live[2, 1] = False
    got = bf16.to_f32(bf16_bits(q)).astype(np.float64)
    assert np.isnan(got[2, 1]).any()
    _, lo, hi = (bf16.to_f32(v) for v in qk.band(ref[live], tol[live]))
    assert ((lo <= got[live]) & (got[live] <= hi)).all()
    check_band(k, *c.forward(1), "k")


@pytest.mark.parametrize("inter", [False, True])
@pytest.mark.parametrize("R", [32, 64])
def test_positions_outside_the_table(P, R, inter):
    import torch
    c = Case(P, 18, 8, 2, 2, 64, R, inter, positions="given")
    good = bf16_bits(P.qk_norm_rope_fwd(c.q, c.k, **c.args)[0])
    bad = c.p_dev.clone()
    bad[2], bad[5], bad[7] = -1, c.rope.table.shape[0], 2 ** 31 - 1
    q, _ = P.qk_norm_rope_fwd(c.q, c.k, **dict(c.args, positions=bad))
    got = bf16_bits(q)
    out = [2, 5, 7]
    keep = [0, 1, 3, 4, 6]
    assert np.isnan(bf16.to_f32(got[out][..., :R])).all()
    assert (got[keep] == good[keep]).all() and (got[out][..., R:] == good[out][..., R:]).all()
    d, _, _ = P.qk_norm_rope_bwd(*c.g, c.q, c.k, **dict(c.args, positions=bad))
    d = bf16.to_f32(bf16_bits(d)).reshape(8, -1, 64)
    assert np.isnan(d[out][:, :4]).any(axis=(1, 2)).all() and not np.isnan(d[keep]).any()
    torch.cuda.synchronize()


# ------------------------------------------------------------------- quantised
RULE = {0: "fp32", 1: "pow2", 2: "pow2_floor"}


def check_quantised(P, c, fmt, mode, r):
    got = P.qk_norm_rope_bwd_quantize_fp8(*c.g, c.q, c.k, fmt=fmt, mode=mode, rnd=r, want_qT=True, **c.args)
    parts = [c.backward(i)[:2] for i in range(2)]
    ref = np.concatenate([p[0] for p in parts] + [f64(c.d[2])], 1).reshape(c.T, -1)
    tol = np.concatenate([p[1] for p in parts] + [np.zeros(c.d[2].shape)], 1).reshape(c.T, -1)
    mid, lo, hi = qk.band(ref, tol)
    un, f, rule = lo == hi, fp8.E4M3 if fmt == E4 else fp8.E5M2, RULE[r]
    km = bool(mode & KMAJOR)
    base = mode & ~KMAJOR
    S = lambda n: host(got[n].t().contiguous() if km else got[n])
    what = "T %d D %d mode %d" % (c.T, c.D, mode)
    if base == TENSOR:
        band_check.check(host(got["q"]), S("scale"), mid, lo, hi, un, f, rule, None, what + " q")
        band_check.check(host(got["qT"]).T, S("scale"), mid, lo, hi, un, f, rule, None, what + " qT")
    if base == ROW:
        band_check.check(host(got["q"]), S("scale"), mid, lo, hi, un, f, rule, 1, what + " q")
    if base in (ROW, COL):
        band_check.check(host(got["qT"]).T, S("scaleT"), mid, lo, hi, un, f, rule, 0, what + " qT")
    check_dgamma(got["dgamma_q"], c, 0, what)
    check_dgamma(got["dgamma_k"], c, 1, what)
    return got


@pytest.mark.parametrize("T,hq,hk,D,R", [(128, 2, 1, 128, 128), (256, 5, 2, 64, 64), (128, 3, 1, 64, 32),
                                         (384, 4, 4, 128, 48)])
@pytest.mark.parametrize("fmt,r", [(E4, 1), (E5, 1), (E4, 2)])
def test_quantised_groups(P, T, hq, hk, D, R, fmt, r):
    c = Case(P, T + D + R, T, hq, hk, D, R, inter=fmt == E5, positions="given")
    cols = (hq + 2 * hk) * D
    if cols % 128 == 0:
        check_quantised(P, c, fmt, ROW, r)
        check_quantised(P, c, fmt, ROW | KMAJOR, r)
    check_quantised(P, c, fmt, COL, r)


@pytest.mark.parametrize("T,hq,hk,D,R,batch", [(16, 1, 1, 64, 64, 1), (144, 3, 1, 64, 32, 3), (208, 2, 1, 128, 128, 1),
                                               (16, 4, 2, 128, 0, 16)])
@pytest.mark.parametrize("fmt,r", [(E5, 0), (E4, 0), (E4, 1)])
def test_quantised_tensor(P, T, hq, hk, D, R, batch, fmt, r):
    check_quantised(P, Case(P, T + hq, T, hq, hk, D, R, inter=hq == 3, batch=batch), fmt, TENSOR, r)


@pytest.mark.parametrize("norm", ["none", "q", "k"])
@pytest.mark.parametrize("D", [64, 128])
def test_quantised_norm_of_one_kind(P, norm, D):
    c = Case(P, 21, 128, 2, 1, D, D, norm=norm)
    check_quantised(P, c, E4, ROW, 1)
    check_quantised(P, c, E4, TENSOR, 0)


def test_quantised_equals_quantising_the_gradient(P):
    """More than one tile in both directions, several sequences: the codes, the scales and dgamma of quantising the
    BF16 gradient, whose arithmetic is the same."""
    import torch
    c = Case(P, 22, 1024, 12, 2, 128, 128, batch=4)
    out, dgq, dgk = P.qk_norm_rope_bwd(*c.g, c.q, c.k, **c.args)
    for mode, r in ((TENSOR, 0), (ROW, 1), (ROW, 2), (COL, 1)):
        want = P.quantize_fp8(out, E4, mode, r, want_qT=True)
        got = P.qk_norm_rope_bwd_quantize_fp8(*c.g, c.q, c.k, fmt=E4, mode=mode, rnd=r, want_qT=True, **c.args)
        for n in ("q", "scale", "qT", "scaleT"):
            assert (want[n] is None) == (got[n] is None) and (want[n] is None or torch.equal(want[n], got[n])), (mode, n)
        for x, y in ((dgq, got["dgamma_q"]), (dgk, got["dgamma_k"])):
            torch.testing.assert_close(x, y, rtol=0, atol=2e-5 * float(x.abs().max()))


@pytest.mark.parametrize("D", [64, 128])
def test_quantised_with_positions_outside_the_table(P, D):
    """In one wave's rows among many: NaN scales and codes of those tokens' turned heads, everything else as it was,
    dgamma NaN."""
    c = Case(P, 28, 256, 3, 1, D, D, positions="given")
    cols, turned = 5 * D, 4 * D
    if cols % 128:
        c = Case(P, 28, 256, 4, 1, D, D, positions="given")
        cols, turned = 6 * D, 5 * D
    run = lambda pos: P.qk_norm_rope_bwd_quantize_fp8(*c.g, c.q, c.k, fmt=E4, mode=ROW, rnd=1,
                                                      **dict(c.args, positions=pos))
    good = run(c.p_dev)
    bad = c.p_dev.clone()
    bad[70], bad[201] = -5, c.rope.table.shape[0] + 3
    got = run(bad)
    keep = np.setdiff1d(np.arange(256), [70, 201])
    q, w = host(got["q"]), host(good["q"])
    assert (q[keep] == w[keep]).all() and (host(got["scale"])[keep] == host(good["scale"])[keep]).all()
    whole = turned // 128                                      # groups of turned heads alone
    assert np.isnan(host(got["scale"])[[70, 201]][:, :whole]).all() and (q[[70, 201]][:, :whole * 128] == 0x7F).all()
    tail = -(-turned // 128) * 128
    assert (q[[70, 201]][:, tail:] == w[[70, 201]][:, tail:]).all()
    assert np.isnan(host(got["dgamma_q"])).all()


@pytest.mark.parametrize("T,batch", [(152, 1), (136, 17), (1032, 3), (200, 25), (8, 1)])
@pytest.mark.parametrize("D", [64, 128])
def test_quantised_ragged_rows(P, T, batch, D):
    """Sequences of whole groups of 8 tokens, and not; rows that end inside a tile; an odd number of heads of 64."""
    c = Case(P, T + D, T, 2, 1, D, D, batch=batch)
    got = P.qk_norm_rope_bwd_quantize_fp8(*c.g, c.q, c.k, fmt=E5, mode=TENSOR, rnd=0, **c.args)
    parts = [c.backward(i)[:2] for i in range(2)]
    ref = np.concatenate([p[0] for p in parts] + [f64(c.d[2])], 1).reshape(T, -1)
    tol = np.concatenate([p[1] for p in parts] + [np.zeros(c.d[2].shape)], 1).reshape(T, -1)
    mid, lo, hi = qk.band(ref, tol)
    band_check.check(host(got["q"]), host(got["scale"]), mid, lo, hi, lo == hi, fp8.E5M2, "fp32", None, "ragged")
    check_dgamma(got["dgamma_q"], c, 0, "ragged")
    check_dgamma(got["dgamma_k"], c, 1, "ragged")


def test_large_offsets(P):
    """Heads more than 2^31 elements after the first one of their tensor."""
    import torch
    c = Case(P, 23, 2, 1, 1, 128, 128)
    far = torch.empty(2 ** 31 + 4096, dtype=torch.bfloat16, device="cuda")
    q = far.as_strided((2, 1, 128), (2 ** 31 + 1024, 128, 1))
    k = far.as_strided((2, 1, 128), (2 ** 31 + 1024, 128, 1), 512)
    q.copy_(c.q)
    k.copy_(c.k)
    c.q, c.k = q, k
    check_forward(P, c, q_out=q, k_out=k)


def test_most_tokens(P):
    """The largest call, 2^25 tokens of one head of 8 (a wave each forward); first, last and drawn tokens against the
    formula in float64. Errors: one rounding to BF16 (2^-8 relative) and a few of 2^-24 of the terms' sizes."""
    import torch
    n, D = 1 << 25, 8
    g = torch.Generator(device="cuda").manual_seed(5)
    x, dy = (torch.randn(n, 1, D, generator=g, device="cuda").to(torch.bfloat16) for _ in range(2))
    gamma = torch.randn(D, generator=g, device="cuda").to(torch.bfloat16)
    none = x[:, :0]
    y, _ = P.qk_norm_rope_fwd(x, none, gamma_q=gamma)
    dx = P.qk_norm_rope_bwd(dy, none, none, x, none, gamma_q=gamma, want_dgamma=False)[0]
    at = torch.cat((torch.arange(1000, device="cuda"), torch.arange(n - 1000, n, device="cuda"),
                    torch.randint(0, n, (100000,), generator=g, device="cuda")))
    xs, ds, gm = x[at, 0].double(), dy[at, 0].double(), gamma.double()
    r = 1 / (xs.square().mean(1, keepdim=True) + 1e-6).sqrt()
    h, gg = xs * r, ds * gm
    ref = h * gm
    assert ((y[at, 0].double() - ref).abs() <= ref.abs() * (2.0 ** -8 + 2.0 ** -18)).all()
    ref, size = r * (gg - h * (gg * h).mean(1, keepdim=True)), r * (gg.abs() + h.abs() * (gg * h).abs().mean(1, keepdim=True))
    assert ((dx[at].double() - ref).abs() <= ref.abs() * 2.0 ** -8 + size * 2.0 ** -18).all()


# ----------------------------------------------------------- streams and graphs
def test_graph_replays_and_another_stream(P):
    """Captured forward and backwards, replayed on changed inputs, against eager calls in between; one workspace per
    captured call."""
    import torch
    c = Case(P, 24, 256, 4, 2, 128, 128)
    q, k = c.q.clone(), c.k.clone()
    g = [v.clone() for v in c.g]

    def step():
        return (*P.qk_norm_rope_fwd(q, k, **c.args), *P.qk_norm_rope_bwd(*g, q, k, **c.args),
                *P.qk_norm_rope_bwd_quantize_fp8(*g, q, k, fmt=E4, mode=TENSOR, want_qT=True, **c.args).values())

    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        step()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=s):
            kept = step()
    torch.cuda.current_stream().wait_stream(s)
    for n in range(4):
        q.copy_(c.q * (n + 1))
        g[0].copy_(c.g[0].flip(0) * (n + 1))
        want = step()
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        for a, b in zip(kept, want):
            assert (a is None and b is None) or torch.equal(a, b)


# ------------------------------------------------------------------- autograd
@pytest.mark.parametrize("batch", [1, 2])
def test_autograd(P, batch):
    import torch
    c = Case(P, 25, 34, 4, 2, 64, 64, batch=batch)
    qkv = dev(c.qkv, batch if batch > 1 else None).requires_grad_(True)
    gq, gk = (c.args[n].clone().requires_grad_(True) for n in ("gamma_q", "gamma_k"))
    q, k, v = P.qk_norm_rope(qkv, 4, 2, gq, gk, c.rope, None, EPS)
    check_band(q, *c.forward(0), "q")
    check_band(k, *c.forward(1), "k")
    torch.autograd.backward((q, k, v), c.g)
    want, dgq, dgk = P.qk_norm_rope_bwd(*c.g, c.q, c.k, **c.args)
    assert torch.equal(qkv.grad.view(34, -1), want)
    assert torch.equal(gq.grad, dgq.to(torch.bfloat16)) and torch.equal(gk.grad, dgk.to(torch.bfloat16))
    # only one of the outputs is used; a gradient of a layout the kernel does not take
    qkv.grad = None
    q, k, v = P.qk_norm_rope(qkv, 4, 2, None, None, c.rope)
    (k.float() * k.float()[..., :1, :].detach()).sum().backward()
    assert qkv.grad is not None and not qkv.grad.view(34, -1)[:, :4 * 64].any()
    assert qkv.grad.view(34, -1)[:, 4 * 64:6 * 64].any() and not qkv.grad.view(34, -1)[:, 6 * 64:].any()


def test_refusals(P):
    import torch
    c = Case(P, 26, 8, 2, 1, 64, 64)
    f = P.qk_norm_rope_fwd
    with pytest.raises(TypeError):
        f(c.q.float(), c.k)
    with pytest.raises(TypeError):
        f(c.q, c.k, rope=c.rope, positions=torch.arange(8, device="cuda"))          # int64
    with pytest.raises(ValueError):
        f(c.q, c.k, rope=c.rope, positions=torch.arange(7, device="cuda", dtype=torch.int32))
    with pytest.raises(ValueError):
        f(c.q, c.k[:-1])
    with pytest.raises(ValueError):
        f(c.q.cpu(), c.k)
    with pytest.raises(ValueError):
        f(c.q.transpose(-1, -2).contiguous().transpose(-1, -2), c.k)
    with pytest.raises(P.PuroError) as e:
        f(c.q[..., :60], c.k[..., :60])
    assert e.value.code == 4
    with pytest.raises(P.PuroError) as e:                                              # all heads in one place
        f(c.q, c.k, q_out=c.q[:, :1].expand(8, 2, 64))
    assert e.value.code == 2
    with pytest.raises(P.PuroError) as e:                                              # 9 positions are too few for 16
        f(c.q.repeat(2, 1, 1), c.k.repeat(2, 1, 1), rope=P.rope_table(9, 64))
    assert e.value.code == 2
    c = Case(P, 27, 128, 2, 1, 32, 32)
    with pytest.raises(P.PuroError) as e:
        P.qk_norm_rope_bwd_quantize_fp8(*c.g, c.q, c.k, mode=ROW, rnd=1, **c.args)     # heads of 32
    assert e.value.code == 3
