"""The query / key norm and the distillation loss as a training step uses them:
FP8 QKV projection -> norm and rotation -> causal attention (torch, binary32)
-> FP8 output projection -> LM head with a teacher's top logits, and back, the
attention's gradients quantised as they pass the norm and multiplied as the
QKV projection's Dgrad and Wgrad. Each new operator's results are checked
against its oracle on the inputs it met there; the quantised way back gives the
bytes of the BF16 gradient's; and autograd gives what the calls give."""

import numpy as np
import pytest

from oracle import bf16, lm_distill as ld, qk_norm_rope as qk
from paper_2608_27370_amd import inputs

from gpu_util import bf16_bits, check_bf16, check_fp32, host, to_dev, to_dev_bf16

pytestmark = pytest.mark.gpu

B, S, K, HQ, HK, D, V, TOP = 2, 128, 256, 4, 2, 64, 1003, 8
T, N = B * S, (HQ + 2 * HK) * D
EPS, TAU = 1e-6, 2.0


@pytest.fixture(scope="module")
def P():
    from paper_2608_27370_amd import puro
    puro.lib()
    return puro


def f64(bits):
    return bf16.to_f32(np.asarray(bits, dtype=np.uint16)).astype(np.float64)


def attention(q, k, v):
    """Causal attention of [B, S, H, D] heads in binary32, key heads shared; [T, HQ D] BF16."""
    import torch
    q, k, v = (t.float().transpose(1, 2).contiguous() for t in (q, k, v))
    k, v = (t.repeat_interleave(HQ // HK, dim=1) for t in (k, v))
    s = (q @ k.transpose(-1, -2).contiguous()) / D ** 0.5
    s = s.masked_fill(torch.ones(S, S, dtype=torch.bool, device=q.device).triu(1), float("-inf"))
    o = s.softmax(-1) @ v
    return o.transpose(1, 2).reshape(T, HQ * D).to(torch.bfloat16)


@pytest.fixture(scope="module")
def step(P):
    """Everything a step reads, and what the calls give one by one."""
    import torch
    g = np.random.default_rng(70)
    s = dict(X=to_dev_bf16(inputs.case(71, (T, K))), Wqkv=to_dev_bf16(inputs.case(72, (N, K), std=0.05)),
             Wo=to_dev_bf16(inputs.case(73, (K, HQ * D), std=0.05)), W=to_dev_bf16(inputs.case(74, (V, K), std=0.05)),
             gq=to_dev_bf16(bf16.from_f64_rne(1 + 0.1 * g.normal(size=D))),
             gk=to_dev_bf16(bf16.from_f64_rne(1 + 0.1 * g.normal(size=D))))
    ids = np.sort(g.integers(0, V, (T, TOP)), axis=1).astype(np.int32)
    ids[100:103] = -1                                          # padding tokens
    teacher = (g.normal(size=(T, TOP)) * 3).astype(np.float32)
    s.update(ids=to_dev(ids), teacher=to_dev(teacher), rope=P.rope_table(S, D, 1e4), recipe=P.LinearRecipe(0, 0, 0, 1, 1),
             ids_host=ids, teacher_host=teacher)
    norm = dict(gamma_q=s["gq"], gamma_k=s["gk"], rope=s["rope"], eps=EPS)
    r = s["recipe"]
    s["qkv"], saved = P.linear_fwd(s["X"], s["Wqkv"], r)
    heads = s["qkv"].view(B, S, HQ + 2 * HK, D)
    q0, k0, v = heads[:, :, :HQ], heads[:, :, HQ:HQ + HK], heads[:, :, HQ + HK:]
    s["q"], s["k"] = P.qk_norm_rope_fwd(q0, k0, **norm)
    leaves = [t.clone().requires_grad_(True) for t in (s["q"], s["k"], v)]
    o = attention(*leaves)
    H, saved_o = P.linear_fwd(o.detach(), s["Wo"], r)
    s["H"] = H
    s["lse"], s["loss"], s["z_top"] = P.lm_head_distill_fwd(H, s["W"], s["ids"], s["teacher"], TAU)
    s["dH"], s["dW"] = P.lm_head_distill_bwd(H, s["W"], s["ids"], s["teacher"], s["lse"], s["z_top"], TAU,
                                             grad_scale=1.0 / T)
    do, s["dWo"] = P.linear_bwd(s["dH"], saved_o, r, HQ * D)
    s["d"] = [t.contiguous() for t in torch.autograd.grad(o, leaves, do)]
    s["dqkv"], s["dgq"], s["dgk"] = P.qk_norm_rope_bwd(*s["d"], q0, k0, **norm)
    s["dX"], s["dWqkv"] = P.linear_bwd(s["dqkv"], saved, r, K)
    # the same with the gradient quantised where it is formed
    mode = P.SCALE_ROW_1x128 | P.SCALE_KMAJOR
    f = s["quantised"] = P.qk_norm_rope_bwd_quantize_fp8(*s["d"], q0, k0, fmt=P.E4M3, mode=mode, rnd=P.SCALE_POW2,
                                                         want_qT=True, **norm)
    s["dX2"] = P.fp8_gemm(P.operand(f["q"], P.E4M3, mode, f["scale"]), T,
                          P.operand(saved["wq_t"], P.E4M3, P.SCALE_BLOCK_128x128 | P.SCALE_KMAJOR, saved["w_scale"]), K, N)
    s["dWqkv2"] = P.fp8_gemm(P.operand(f["qT"], P.E4M3, mode, f["scaleT"]), N,
                             P.operand(saved["xq_t"], P.E4M3, mode, saved["x_scale"]), K, T, out_dtype=P.OUT_FP32)
    return s


def test_norm_and_rotation_on_what_they_met(step):
    x = f64(bf16_bits(step["qkv"])).reshape(T, HQ + 2 * HK, D)
    table = host(step["rope"].table).astype(np.float64)
    cos, sin = np.tile(table[..., 0], (B, 1)), np.tile(table[..., 1], (B, 1))
    dqkv = bf16.to_f32(bf16_bits(step["dqkv"])).reshape(T, HQ + 2 * HK, D)
    for lo, hi, gamma, y, dy, dgamma in ((0, HQ, "gq", "q", 0, "dgq"), (HQ, HQ + HK, "gk", "k", 1, "dgk")):
        gm = f64(bf16_bits(step[gamma]))
        ref, tol = qk.forward(x[:, lo:hi], gm, EPS, cos, sin)
        got = bf16.to_f32(bf16_bits(step[y])).reshape(ref.shape)
        _, a, b = (bf16.to_f32(t) for t in qk.band(ref, tol))
        assert ((a <= got) & (got <= b)).all()
        d = f64(bf16_bits(step["d"][dy])).reshape(ref.shape)
        ref, tol, dref, dtol = qk.backward(d, x[:, lo:hi], gm, EPS, cos, sin)
        _, a, b = (bf16.to_f32(t) for t in qk.band(ref, tol))
        assert ((a <= dqkv[:, lo:hi]) & (dqkv[:, lo:hi] <= b)).all()
        assert (np.abs(host(step[dgamma]) - dref) <= dtol).all()
    assert (dqkv[:, HQ + HK:] == f64(bf16_bits(step["d"][2])).reshape(T, HK, D)).all()


def test_loss_on_what_it_met(step):
    H, W = bf16_bits(step["H"]), bf16_bits(step["W"])
    f = ld.forward(H, W, step["ids_host"], step["teacher_host"], TAU, ld.LOGITS)
    for n, t in (("lse", "tol_lse"), ("loss", "tol_loss"), ("z_top", "tol_z")):
        assert (np.abs(host(step[n]) - f[n]) <= f[t] + 2.0 ** -24 * np.abs(f[n])).all(), n
    assert not host(step["loss"])[100:103].any() and not bf16_bits(step["dH"])[100:103].any()
    mid, lo, hi = (f64(v) for v in ld.dz_band(f, TAU, np.ones(T), 1.0 / T))
    h, w = f64(H), f64(W)
    check_bf16(bf16_bits(step["dH"]), mid @ w, np.abs(mid) @ np.abs(w), what="dH", slack=(hi - lo) @ np.abs(w))
    check_fp32(host(step["dW"]), mid.T @ h, np.abs(mid).T @ np.abs(h), what="dW", slack=(hi - lo).T @ np.abs(h))


def test_the_quantised_way_back_gives_the_same_bytes(step):
    import torch
    assert torch.equal(step["dX"], step["dX2"]) and torch.equal(step["dWqkv"], step["dWqkv2"])


def test_autograd_gives_what_the_calls_give(P, step):
    import torch
    s = step
    X = s["X"].clone().requires_grad_(True)
    Wqkv, Wo, W, gq, gk = (torch.nn.Parameter(s[n].clone()) for n in ("Wqkv", "Wo", "W", "gq", "gk"))
    for w in (Wqkv, Wo, W):
        w.main_grad = torch.zeros(w.shape, device="cuda")
    qkv = P.linear(X.view(B, S, K), Wqkv, s["recipe"])
    o = attention(*P.qk_norm_rope(qkv, HQ, HK, gq, gk, s["rope"], None, EPS))
    loss = P.lm_head_distill(P.linear(o, Wo, s["recipe"]), W, s["ids"], s["teacher"], TAU)
    assert torch.equal(loss, s["loss"])
    (loss * (1.0 / T)).sum().backward()
    # the upstream gradient of each loss is 1 / T here, and a factor of ones there: the same products
    assert torch.equal(W.main_grad, s["dW"]) and torch.equal(Wo.main_grad, s["dWo"])
    assert torch.equal(X.grad, s["dX"]) and torch.equal(Wqkv.main_grad, s["dWqkv"])
    assert torch.equal(gq.grad, s["dgq"].to(torch.bfloat16)) and torch.equal(gk.grad, s["dgk"].to(torch.bfloat16))
