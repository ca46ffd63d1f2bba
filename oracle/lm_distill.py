"""The language-model head with the divergence from a teacher's top logits as
its loss, forward and backward, in float64.

Test infrastructure only (see the package docstring). The head is the one of
oracle/lm_head.py (BF16 operands); the loss is the usual distillation one, a
teacher known by k entries (id, value) per token:

    z = X W^T, a = z / tau, lse = log sum_v exp(a_v)
    q = softmax of the entries' values over tau, or the values themselves
    loss = sum_j q_j (log q_j - a_{id_j} + lse)
    dz_v = dloss g / tau (Q exp(a_v - lse) - sum_{j: id_j = v} q_j),  Q = sum_j q_j

over the entries whose id lies in [0, V). The readings: q, the statistics and
the sums in binary32, each logit of the loss a binary32 sum, dz rounded once to
BF16.

Allowances of a binary32 evaluation, u = 2^-24:
  * a: TOL_Z sum_k |x_k w_k| / tau + 2 u |a| (the GEMM's sum, the quotient by way
    of 1 / tau); z_top: TOL_Z sum |x w| (a sum at most K / 64 + 14 deep);
  * lse: its row's largest logit allowance plus LSE_ABS (1 + |lse|);
  * log q (LOGITS): the difference (t - top) / tau errs by 3 u of its size, the
    log of the sum by its terms' errors and a few u: Q_REL (1 + |log q|) with
    Q_REL = 2^-20; q: that, relative, plus 4 u (exp);
  * loss: sum_j q_j (the allowances of log q, a, lse and their sum's rounding)
    plus q's relative allowance times |log q - a + lse|;
  * dz: the dense part relative by exp's (the allowances of a and lse plus
    EXP_REL) and q's; an entry's sum of q by q's.

Parity unpinned by the paper (it distils nothing); pinned in
tests/test_oracle_lm_distill.py by finite differences, by scipy's relative
entropy and by closed forms.
"""

import numpy as np

from . import bf16
from .lm_head import EXP_REL, LSE_ABS, TOL_Z, logits

Q_REL = 2.0 ** -20
LOGITS, PROBS = 0, 1


def teacher(ids, values, V, tau, kind):
    """(q, log q where q > 0 else 0, allowance of log q), float64 [M, k]."""
    ok = (ids >= 0) & (ids < V)
    t = values.astype(np.float64)
    with np.errstate(divide="ignore", invalid="ignore", over="ignore"):
        if kind == PROBS:
            q = np.where(ok, t, 0.0)
            log_q = np.where(q > 0, np.log(np.where(q > 0, q, 1.0)), 0.0)
        else:
            t = np.where(ok, t, -np.inf)
            top = t.max(axis=1, keepdims=True)
            d = np.where(top > -np.inf, (t - top) / tau, -np.inf)
            log_q = d - np.log(np.exp(d).sum(axis=1, keepdims=True))
            q = np.where(ok & (top > -np.inf), np.exp(log_q), 0.0)
            log_q = np.where(q > 0, log_q, 0.0)
    return q, log_q, Q_REL * (1.0 + np.abs(log_q))


def forward(X_bits, W_bits, ids, values, tau, kind):
    """dict of lse, loss, z_top and their allowances, and what the backward takes."""
    z, S = logits(X_bits, W_bits)
    V = z.shape[1]
    a, tol_a = z / tau, TOL_Z * S / tau + 2.0 ** -23 * np.abs(z / tau)
    top = a.max(axis=1)
    lse = top + np.log(np.exp(a - top[:, None]).sum(axis=1))
    tol_lse = tol_a.max(axis=1) + LSE_ABS * (1.0 + np.abs(lse))
    ok = (ids >= 0) & (ids < V)
    at = np.where(ok, ids, 0)
    z_top = np.where(ok, np.take_along_axis(z, at, 1), 0.0)
    tol_z = np.where(ok, TOL_Z * np.take_along_axis(S, at, 1), 0.0)
    q, log_q, tol_q = teacher(ids, values, V, tau, kind)
    term = log_q - z_top / tau + lse[:, None]
    loss = (q * term).sum(axis=1)
    each = tol_q + tol_z / tau + tol_lse[:, None] + 2.0 ** -21 * (np.abs(log_q) + np.abs(z_top / tau) + np.abs(lse)[:, None])
    tol_loss = (q * (each + (tol_q + 2.0 ** -21) * np.abs(term))).sum(axis=1)
    return dict(a=a, tol_a=tol_a, lse=lse, tol_lse=tol_lse, loss=loss, tol_loss=tol_loss, z_top=z_top, tol_z=tol_z, q=q,
                tol_q=tol_q, ok=ok, at=at)


def dz_band(f, tau, dloss, grad_scale):
    """BF16 patterns (mid, lo, hi) [M, V] of dz of grad_scale sum dloss loss."""
    g = (dloss * np.float64(np.float32(grad_scale)) / tau)[:, None]
    q = np.where(f["ok"], f["q"], 0.0)
    e = g * q.sum(axis=1, keepdims=True) * np.exp(f["a"] - f["lse"][:, None])
    rel_q = f["tol_q"] + 2.0 ** -21
    tol = np.abs(e) * (f["tol_a"] + f["tol_lse"][:, None] + EXP_REL + rel_q.max(axis=1, keepdims=True))
    dz, rows = e.copy(), np.arange(e.shape[0])[:, None]
    np.add.at(dz, (rows, f["at"]), -g * q)
    np.add.at(tol, (rows, f["at"]), np.abs(g) * q * (rel_q + 2.0 ** -20))
    tol = tol + 2.0 ** -140
    return bf16.from_f64_rne(dz), bf16.from_f64_rne(dz - tol), bf16.from_f64_rne(dz + tol)


def gradient(X_bits, W_bits, ids, values, tau, kind, dloss, grad_scale=1.0):
    """dz [M, V] in float64 without any rounding (for differences)."""
    f = forward(X_bits, W_bits, ids, values, tau, kind)
    g = (dloss * grad_scale / tau)[:, None]
    dz = g * f["q"].sum(axis=1, keepdims=True) * np.exp(f["a"] - f["lse"][:, None])
    np.add.at(dz, (np.arange(dz.shape[0])[:, None], f["at"]), -g * np.where(f["ok"], f["q"], 0.0))
    return dz
