"""The query/key norms with their position rotation, and the LM head's distillation loss, as cases to time and compare.

Each case is one pass through an operator of ``paper_2608_27370_amd.puro`` (``own``), or the same operator in plain
torch operations in binary32, rounded once at the end. Operators (``op``):

* ``rope_fwd``    -- RMSNorm of every query and key head and the position rotation, from the fused QKV projection's output.
* ``rope_bwd``    -- its backward: the gradient of the projection's output (the value heads' included) and of both weights.
* ``rope_bwd_q``  -- the backward with the gradient quantised to FP8 as the projection's Dgrad and Wgrad read it.
* ``distill_fwd`` -- LM head with the divergence from a teacher's top logits as its loss, the logits not stored.
* ``distill_bwd`` -- its backward: the gradients of the hidden states and of the output embedding.

Sizes are those of the paper's 1.7B model (16 query and 8 key heads of 128, hidden size 2048) and of Qwen2-1.5B
(12 and 2 heads of 128, hidden size 1536, 151936 tokens), and generic ones around them.
"""

import math

import torch

own = False

G = 128
EPS = 1e-6


def listed():
    return [
        # one token of one sequence, far into its context: the smallest call
        dict(name="rope_fwd_decode_1", op="rope_fwd", B=1, S=1, Hq=12, Hk=2, D=128, R=128, inter=False, norm=True,
             pos="far", L=131072, heads_first=False),
        # a short ragged batch, heads of 64 with interleaved pairs, half of each head rotated, no norm
        dict(name="rope_fwd_partial_777", op="rope_fwd", B=1, S=777, Hq=9, Hk=3, D=64, R=32, inter=True, norm=False,
             pos="packed", L=4096, heads_first=False),
        # two packed 4096-token sequences of the 1.7B model, written heads first as attention may want them
        dict(name="rope_fwd_8192", op="rope_fwd", B=2, S=4096, Hq=16, Hk=8, D=128, R=128, inter=False, norm=True,
             pos="rows", L=4096, heads_first=True),
        # the same micro-batch's backward, gradients heads first as attention gives them
        dict(name="rope_bwd_8192", op="rope_bwd", B=2, S=4096, Hq=16, Hk=8, D=128, R=128, inter=False, norm=True,
             pos="rows", L=4096, heads_first=True),
        # an odd number of tokens, heads of 80 of which 64 are rotated
        dict(name="rope_bwd_odd_1531", op="rope_bwd", B=1, S=1531, Hq=10, Hk=5, D=80, R=64, inter=False, norm=True,
             pos="packed", L=8192, heads_first=False),
        # the paper's blockwise recipe: both quantised copies of the QKV projection's output gradient
        dict(name="rope_bwd_q_block_8192", op="rope_bwd_q", B=2, S=4096, Hq=16, Hk=8, D=128, R=128, inter=False,
             norm=True, pos="rows", L=4096, heads_first=False, blockwise=True),
        # per-tensor scales at the Qwen2-1.5B heads, a small micro-batch
        dict(name="rope_bwd_q_tensor_1024", op="rope_bwd_q", B=1, S=1024, Hq=12, Hk=2, D=128, R=128, inter=False,
             norm=True, pos="rows", L=4096, heads_first=False, blockwise=False),
        # a short ragged batch over a small vocabulary, odd sizes everywhere
        dict(name="distill_fwd_77", op="distill_fwd", M=77, V=5003, K=520, topk=7, tau=2.0, target="logits"),
        # the full vocabulary at half a micro-batch, the teacher's 64 best tokens
        dict(name="distill_fwd_4096", op="distill_fwd", M=4096, V=151936, K=1536, topk=64, tau=1.0, target="logits"),
        # a GPT-2-sized odd vocabulary, probabilities as stored by a teacher's run
        dict(name="distill_bwd_1000", op="distill_bwd", M=1000, V=50257, K=1024, topk=20, tau=1.0, target="probs"),
        # the largest: one 8192-token micro-batch's backward over the full vocabulary
        dict(name="distill_bwd_8192", op="distill_bwd", M=8192, V=151936, K=1536, topk=64, tau=2.0, target="logits"),
    ]


def _log(rng, lo, hi, step=1):
    """A size between lo and hi, even over its logarithm, a multiple of step."""
    v = math.exp(rng.uniform(math.log(lo), math.log(hi)))
    return max(-(-lo // step) * step, min(hi // step * step, int(round(v / step)) * step))


def draw(rng):
    op = rng.choice(["rope_fwd", "rope_fwd", "rope_bwd", "rope_bwd", "rope_bwd_q", "distill_fwd", "distill_bwd"])
    if op.startswith("distill"):
        return dict(op=op, M=_log(rng, 1, 6000), V=_log(rng, 1000, 151936), K=_log(rng, 256, 1536, 8),
                    topk=_log(rng, 1, 64), tau=rng.choice([1.0, 0.7, 2.0, 4.0]), target=rng.choice(["logits", "probs"]))
    quant = op == "rope_bwd_q"
    D = rng.choice([64, 128]) if quant else rng.choice([64, 80, 96, 128, 128, 128, 192, 256])
    Hk = rng.choice([1, 2, 3, 4, 8])
    Hq = Hk * rng.choice([1, 2, 3, 4] if D > 128 else [1, 2, 4, 6])
    blockwise = quant and rng.random() < 0.6
    B = rng.choice([1, 1, 2, 3])
    S = max(1, _log(rng, 1, 8192) // B)
    if quant:
        S = -(-S // (G if blockwise else 16)) * (G if blockwise else 16)
        Hq += (Hq + 2 * Hk) % 2                     # whole 128-column groups
    R = rng.choice([D, D, D // 32 * 16, 0])
    case = dict(op=op, B=B, S=S, Hq=Hq, Hk=Hk, D=D, R=R, inter=rng.random() < 0.3, norm=R == 0 or rng.random() < 0.75,
                pos=rng.choice(["rows", "packed", "far"]), L=rng.choice([8192, 32768]), heads_first=rng.random() < 0.4)
    return dict(case, blockwise=blockwise) if quant else case


# ------------------------------------------------------------------- inputs
def _gen(seed, t):
    return torch.Generator(device="cuda").manual_seed(seed * 16 + t)


def _normal(seed, t, shape, std=1.0, dtype=torch.bfloat16):
    return (torch.randn(shape, generator=_gen(seed, t), device="cuda") * std).to(dtype)


def _positions(c, seed):
    """int32 positions of the B S tokens: each sequence from 0 ("rows": none given), packed documents, far ones."""
    n = c["B"] * c["S"]
    i = torch.arange(n, device="cuda", dtype=torch.int64)
    if c["pos"] == "packed":
        at = torch.randint(0, max(1, n), (max(1, n // 300),), generator=_gen(seed, 1), device="cuda")
        starts = torch.zeros(n, dtype=torch.int64, device="cuda").scatter_(0, at, at)
        return ((i - starts.cummax(0).values) % c["L"]).to(torch.int32)
    if c["pos"] == "far":
        return torch.randint(c["L"] // 2, c["L"], (n,), generator=_gen(seed, 1), device="cuda", dtype=torch.int32)
    return None


def _angles(c):
    """Rotation angles of positions [0, L) in 64 bits: p theta^(-2 i / R), theta = 10^6."""
    i = torch.arange(c["R"] // 2, device="cuda", dtype=torch.float64)
    return torch.arange(c["L"], device="cuda", dtype=torch.float64)[:, None] * 1e6 ** (-2.0 * i / max(1, c["R"]))


def _heads(c, seed, t, h):
    """A gradient of h heads [B, S, h, D] as attention's backward gives it: token by token, or heads first."""
    shape = (c["B"], h, c["S"], c["D"]) if c["heads_first"] else (c["B"], c["S"], h, c["D"])
    x = _normal(seed, t, shape, 1e-3)
    return x.transpose(1, 2) if c["heads_first"] else x


def _prepare_rope(c, seed):
    Hq, Hk, D = c["Hq"], c["Hk"], c["D"]
    C = (Hq + 2 * Hk) * D
    # the projection's output: every channel with a scale of its own, as norms of queries and keys meet it
    scale = torch.exp(torch.randn(C, generator=_gen(seed, 2), device="cuda"))
    s = dict(case=c, qkv=(torch.randn((c["B"], c["S"], C), generator=_gen(seed, 3), device="cuda") * scale).to(torch.bfloat16),
             positions=_positions(c, seed), gq=None, gk=None, table=None)
    if c["norm"]:
        s["gq"] = (1 + 0.1 * torch.randn(D, generator=_gen(seed, 4), device="cuda")).to(torch.bfloat16)
        s["gk"] = (1 + 0.1 * torch.randn(D, generator=_gen(seed, 5), device="cuda")).to(torch.bfloat16)
    if c["R"]:
        a = _angles(c)
        s["table"] = torch.stack((a.cos(), a.sin()), dim=-1).to(torch.float32)       # [L, R / 2, 2]
    if c["op"] != "rope_fwd":
        s.update(dq=_heads(c, seed, 6, Hq), dk=_heads(c, seed, 7, Hk), dv=_heads(c, seed, 8, Hk))
    return s


def _prepare_distill(c, seed):
    M, V, K, k = c["M"], c["V"], c["K"], c["topk"]
    g = _gen(seed, 1)
    # heavy-tailed hidden states, as at the LM head (Student-t with 3 degrees of freedom)
    z = torch.randn((M, K), generator=g, device="cuda")
    chi = sum(torch.randn((M, K), generator=g, device="cuda").square_() for _ in range(3))
    # the teacher's best tokens, frequent (low) ids more often than rare ones; a repeated id and what lies past the
    # teacher's list are marked -1, and so are all entries of a padding token
    ids = (V * torch.rand((M, k), generator=g, device="cuda", dtype=torch.float64) ** 4).to(torch.int64).clamp_(max=V - 1)
    srt = ids.sort(dim=1)
    again = torch.zeros_like(ids, dtype=torch.bool)
    again.scatter_(1, srt.indices[:, 1:], srt.values[:, 1:] == srt.values[:, :-1])
    pad = torch.rand((M, 1), generator=g, device="cuda") < 0.03
    pad[0] = False
    rank = torch.arange(k, device="cuda", dtype=torch.float32)
    t = 14.0 - 2.0 * torch.log1p(rank) + 0.5 * torch.randn((M, k), generator=g, device="cuda")
    if c["target"] == "probs":
        t = torch.softmax(t, dim=1) * (0.75 + 0.2 * torch.rand((M, 1), generator=g, device="cuda"))
    s = dict(case=c, X=(z / (chi / 3.0).sqrt()).to(torch.bfloat16), W=_normal(seed, 2, (V, K), 0.02),
             ids=torch.where(again | pad, -1, ids).to(torch.int32), teacher=t)
    if c["op"] == "distill_bwd":
        # the gradient of the mean over the tokens that count, and what the forward pass kept
        live = (s["ids"] >= 0).any(dim=1)
        s["dloss"] = torch.where(live, 1.0, 0.0) / max(1.0, float(live.sum()))
        _, s["lse"], s["z_top"] = _distill_fwd(s)[1]
        s["dX"] = torch.empty_like(s["X"])
        s["dW"] = torch.empty_like(s["W"])
    return s


def prepare(case, seed):
    return _prepare_distill(case, seed) if case["op"].startswith("distill") else _prepare_rope(case, seed)


# -------------------------------------------------------------- plain forms
def _rotate(x, s, back=False):
    """The rotation of the pairs of x [B, S, H, D] by the table's angles (back: by their negatives)."""
    c = s["case"]
    R, h = c["R"], c["R"] // 2
    if not R:
        return x
    p = s["positions"]
    cs = s["table"][p.long()].view(c["B"], c["S"], 1, h, 2) if p is not None else s["table"][: c["S"]].view(1, c["S"], 1, h, 2)
    cos, sin = cs[..., 0], -cs[..., 1] if back else cs[..., 1]
    a, b = (x[..., 0:R:2], x[..., 1:R:2]) if c["inter"] else (x[..., :h], x[..., h:R])
    u, v = a * cos - b * sin, b * cos + a * sin
    turned = torch.stack((u, v), dim=-1).flatten(-2) if c["inter"] else torch.cat((u, v), dim=-1)
    return torch.cat((turned, x[..., R:]), dim=-1)


def _split(s):
    c = s["case"]
    x = s["qkv"].view(c["B"], c["S"], c["Hq"] + 2 * c["Hk"], c["D"])
    return x[:, :, :c["Hq"]], x[:, :, c["Hq"]:c["Hq"] + c["Hk"]]


def _norm_rope(x, gamma, s):
    x = x.float()
    if gamma is not None:
        x = x * (1.0 / (x.square().mean(dim=-1, keepdim=True) + EPS).sqrt()) * gamma.float()
    return _rotate(x, s).to(torch.bfloat16)


def _norm_rope_bwd(dy, x, gamma, s):
    """The gradients of a head's input and of the weight."""
    dn = _rotate(dy.float(), s, back=True)
    if gamma is None:
        return dn, None
    x = x.float()
    r = 1.0 / (x.square().mean(dim=-1, keepdim=True) + EPS).sqrt()
    xh = x * r
    dgamma = (dn * xh).sum(dim=(0, 1, 2), dtype=torch.float64).float()
    g = dn * gamma.float()
    return r * (g - xh * (g * xh).mean(dim=-1, keepdim=True)), dgamma


def _rope_bwd(s):
    c = s["case"]
    q, k = _split(s)
    dq, dgq = _norm_rope_bwd(s["dq"], q, s["gq"], s)
    dk, dgk = _norm_rope_bwd(s["dk"], k, s["gk"], s)
    dqkv = torch.cat((dq, dk, s["dv"].float()), dim=2).to(torch.bfloat16)
    return dqkv.view(c["B"] * c["S"], -1), dgq, dgk


def _values(codes, scale):
    """What FP8 codes stand for, in BF16 (which holds a code times a power of two exactly)."""
    v = codes.view(torch.float8_e4m3fn).to(torch.bfloat16)
    if scale.numel() == 1:
        return v * scale.to(torch.float32)
    return (v.view(v.shape[0], -1, G) * scale.to(torch.bfloat16)[..., None]).view(v.shape)


def _quantize_groups(x):
    """E4M3 codes and power-of-two scales of groups of 128 along the rows of a BF16 matrix."""
    v = x.float().view(x.shape[0], -1, G)
    m, e = torch.frexp(v.abs().amax(dim=-1))                # amax = m 2^e, 1/2 <= m < 1; the largest code is 7/8 2^9
    e = torch.where(m == 0, 0, e - 9 + (m > 0.875).to(e.dtype)).to(torch.int32)
    power = lambda n: ((n + 127) << 23).view(torch.float32)         # noqa: E731 (2^n; a power that rounds would break ties)
    codes = (v * power(-e)[..., None]).to(torch.float8_e4m3fn)
    return codes.view(x.shape), power(e)


def _rope_bwd_q(s):
    dqkv, dgq, dgk = _rope_bwd(s)
    if s["case"]["blockwise"]:
        q, scale = _quantize_groups(dqkv)
        qT, scaleT = _quantize_groups(dqkv.t().contiguous())
    else:
        amax = dqkv.float().abs().amax()
        scale = scaleT = amax / 448.0
        q = (dqkv.float() * (448.0 / amax)).to(torch.float8_e4m3fn)
        qT = q.view(torch.uint8).t().contiguous().view(torch.float8_e4m3fn)
    return _values(q, scale), _values(qT, scaleT), dgq, dgk


def _targets(s):
    """Which entries count, and the teacher's weights of all of them (0 where they do not)."""
    c = s["case"]
    ok = (s["ids"] >= 0) & (s["ids"] < c["V"])
    if c["target"] == "probs":
        return ok, torch.where(ok, s["teacher"], 0.0)
    t = torch.where(ok, s["teacher"], -math.inf)
    top = t.amax(dim=1, keepdim=True)
    e = torch.where(ok, torch.exp((t - top) / c["tau"]), 0.0)
    return ok, e / e.sum(dim=1, keepdim=True).clamp_min(1e-30)


def _distill_fwd(s):
    """(logits over the temperature, (loss, lse, z_top))."""
    c = s["case"]
    z = s["X"].float() @ s["W"].float().t()
    ok, q = _targets(s)
    z_top = torch.where(ok, z.gather(1, s["ids"].clamp_min(0).long()), 0.0)
    a = z.div_(c["tau"])
    top = a.amax(dim=1, keepdim=True)
    lse = (top + torch.exp(a - top).sum(dim=1, keepdim=True).log()).squeeze(1)
    log_q = torch.where(q > 0, q, 1.0).log()
    loss = (q * (log_q - z_top / c["tau"] + lse[:, None])).sum(dim=1)
    return a, (loss, lse, z_top)


def _distill_bwd(s):
    c = s["case"]
    a = s["X"].float() @ s["W"].float().t()
    a.div_(c["tau"])
    ok, q = _targets(s)
    g = s["dloss"][:, None] / c["tau"]
    dz = a.sub_(s["lse"][:, None]).exp_().mul_(g * q.sum(dim=1, keepdim=True))
    dz.scatter_add_(1, s["ids"].clamp_min(0).long(), -g * q)
    return (dz @ s["W"].float()).to(torch.bfloat16), (dz.t() @ s["X"].float()).to(torch.bfloat16)


# ---------------------------------------------------------------- the calls
def _own_rope(s):
    from paper_2608_27370_amd import puro as P
    c = s["case"]
    q, k = _split(s)
    rope = P.Rope(s["table"], interleaved=c["inter"]) if c["R"] else None
    args = dict(gamma_q=s["gq"], gamma_k=s["gk"], rope=rope, positions=s["positions"], eps=EPS)
    if c["op"] == "rope_fwd":
        if c["heads_first"]:
            args.update(q_out=torch.empty((c["B"], c["Hq"], c["S"], c["D"]), dtype=q.dtype, device=q.device).transpose(1, 2),
                        k_out=torch.empty((c["B"], c["Hk"], c["S"], c["D"]), dtype=q.dtype, device=q.device).transpose(1, 2))
        return P.qk_norm_rope_fwd(q, k, **args)
    if c["op"] == "rope_bwd":
        return P.qk_norm_rope_bwd(s["dq"], s["dk"], s["dv"], q, k, **args)
    mode, rnd = (P.SCALE_ROW_1x128, P.SCALE_POW2) if c["blockwise"] else (P.SCALE_TENSOR, P.SCALE_FP32)
    r = P.qk_norm_rope_bwd_quantize_fp8(s["dq"], s["dk"], s["dv"], q, k, fmt=P.E4M3, mode=mode, rnd=rnd, want_qT=True, **args)
    scale, scaleT = (r["scale"], r["scaleT"]) if c["blockwise"] else (r["scale"][0], r["scale"][0])
    return _values(r["q"], scale), _values(r["qT"], scaleT), r["dgamma_q"], r["dgamma_k"]


def _own_distill(s):
    from paper_2608_27370_amd import puro as P
    c = s["case"]
    kind = P.DISTILL_LOGITS if c["target"] == "logits" else P.DISTILL_PROBS
    if c["op"] == "distill_fwd":
        lse, loss, z_top = P.lm_head_distill_fwd(s["X"], s["W"], s["ids"], s["teacher"], temperature=c["tau"], target=kind)
        return loss, lse, z_top
    return P.lm_head_distill_bwd(s["X"], s["W"], s["ids"], s["teacher"], s["lse"], s["z_top"], temperature=c["tau"],
                                 target=kind, dloss=s["dloss"], dX=s["dX"], dW=s["dW"])


def run(state):
    op = state["case"]["op"]
    if own:
        return _own_distill(state) if op.startswith("distill") else _own_rope(state)
    if op == "rope_fwd":
        q, k = _split(state)
        return _norm_rope(q, state["gq"], state), _norm_rope(k, state["gk"], state)
    if op == "distill_fwd":
        return _distill_fwd(state)[1]
    return {"rope_bwd": _rope_bwd, "rope_bwd_q": _rope_bwd_q, "distill_bwd": _distill_bwd}[op](state)


def work(case):
    if case["op"].startswith("distill"):
        M, V, K, k = (case[n] for n in ("M", "V", "K", "topk"))
        entries = M * k * 8
        if case["op"] == "distill_fwd":
            return {"bytes": 2 * (M + V) * K + entries + M * k * 4 + M * 8, "flops": 2.0 * M * V * K}
        return {"bytes": 4 * (M + V) * K + entries + M * k * 4 + M * 8, "flops": 6.0 * M * V * K}
    T, D, Hq, Hk = case["B"] * case["S"], case["D"], case["Hq"], case["Hk"]
    n, nv = T * (Hq + Hk) * D, T * Hk * D
    seen = T if case["pos"] != "rows" else case["S"]
    side = min(seen, case["L"]) * case["R"] * 4 + (T * 4 if case["pos"] != "rows" else 0) + (4 * D if case["norm"] else 0)
    if case["op"] == "rope_fwd":
        return {"bytes": 4 * n + side, "flops": 10.0 * n}
    reads = 2 * n + 2 * nv + (2 * n if case["norm"] else 0)
    writes = 2 * (n + nv)          # BF16, or both FP8 copies
    return {"bytes": reads + writes + side + (8 * D if case["norm"] else 0), "flops": 20.0 * n}


# ------------------------------------------------- the definition, in 64 bits
def _turn64(x, c, angle):
    """Each pair as a complex number, turned by e^(i angle); x [B, S, H, D], angle [B or 1, S, 1, R / 2]."""
    R = c["R"]
    if not R:
        return x
    head, rest = x[..., :R], x[..., R:]
    pairs = head.unflatten(-1, (R // 2, 2)) if c["inter"] else head.unflatten(-1, (2, R // 2)).transpose(-1, -2)
    z = torch.view_as_complex(pairs.contiguous()) * torch.polar(torch.ones_like(angle), angle)
    out = torch.view_as_real(z)
    out = out.flatten(-2) if c["inter"] else out.transpose(-1, -2).flatten(-2)
    return torch.cat((out, rest), dim=-1)


def _exact_rope(c, seed):
    s = prepare(c, seed)
    B, S, Hq, Hk, D = (c[n] for n in ("B", "S", "Hq", "Hk", "D"))
    p = s["positions"].double().view(B, S) if s["positions"] is not None else torch.arange(S, device="cuda").double()[None]
    i = torch.arange(c["R"] // 2, device="cuda", dtype=torch.float64)
    angle = (p[..., None] * torch.exp(-2.0 * i * math.log(1e6) / max(1, c["R"])))[:, :, None]
    x = s["qkv"].double().view(B, S, -1, D)
    bwd = c["op"] != "rope_fwd"
    outs, grads = [], []
    for lo, hi, gamma, dy in ((0, Hq, s["gq"], s.get("dq")), (Hq, Hq + Hk, s["gk"], s.get("dk"))):
        xx = x[:, :, lo:hi].clone().requires_grad_(bwd)
        n = xx
        if gamma is not None:
            gamma = gamma.double().requires_grad_(bwd)
            n = xx * gamma / torch.sqrt((xx * xx).sum(-1, keepdim=True) / D + EPS)
        y = _turn64(n, c, angle)
        outs.append(y)
        if bwd:
            grads.append(torch.autograd.grad(y, (xx,) if gamma is None else (xx, gamma), dy.double()))
    if not bwd:
        return tuple(outs)
    dqkv = torch.cat([g[0] for g in grads] + [s["dv"].double()], dim=2).reshape(B * S, -1)
    dgq, dgk = (g[1] if len(g) > 1 else None for g in grads)
    if c["op"] == "rope_bwd":
        return dqkv, dgq, dgk
    v = dqkv.to(torch.bfloat16).double()
    near = lambda u: u.float().to(torch.float8_e4m3fn).double()          # noqa: E731 (the nearest code's value)
    if not c["blockwise"]:
        unit = v.abs().max() / 448.0
        w = near(v / unit) * unit
        return w, w.t(), dgq, dgk

    def grouped(m):
        u = m.unflatten(-1, (-1, G))
        top = u.abs().amax(-1, keepdim=True) / 448.0        # the least power of two that is not below it
        n = torch.floor(torch.log2(top.clamp_min(1e-30))).to(torch.int64) - 1
        unit = ((n + 1023) << 52).view(torch.float64)
        for _ in range(3):
            unit = torch.where(unit < top, unit * 2.0, unit)
        return (near(u / unit) * unit).flatten(-2)
    return grouped(v), grouped(v.t().contiguous()), dgq, dgk


def _exact_distill(c, seed):
    s = prepare(c, seed)
    X, W = s["X"].double(), s["W"].double()
    bwd = c["op"] == "distill_bwd"
    a = ((X @ W.t()) / c["tau"]).requires_grad_(bwd)
    lse = torch.logsumexp(a, dim=1)
    ok = (s["ids"] >= 0) & (s["ids"] < c["V"])
    at = torch.where(ok, s["ids"], 0).long()
    t = s["teacher"].double()
    if c["target"] == "logits":
        t = torch.softmax(torch.where(ok, t / c["tau"], -1e300), dim=1)
    q = t * ok
    picked = a.gather(1, at)
    loss = (torch.special.xlogy(q, q) - q * (picked - lse[:, None])).sum(dim=1)
    if not bwd:
        return loss, lse, torch.where(ok, picked * c["tau"], 0.0)
    (da,) = torch.autograd.grad(loss, a, s["dloss"].double())
    dz = da / c["tau"]
    return dz @ W, dz.t() @ X


def exact(case, seed):
    return _exact_distill(case, seed) if case["op"].startswith("distill") else _exact_rope(case, seed)
