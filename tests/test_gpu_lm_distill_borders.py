"""The distillation backward at the borders of its parts: between the chunks of
a large vocabulary, with entries on both sides of every border, and in the
products for dX over a long vocabulary, split in 256 x 192 tiles."""

import numpy as np
import pytest

from oracle import lm_distill as ld

from gpu_util import check_fp32, host, to_dev
from test_gpu_lm_distill import L, Case, check_forward, check_gradients, f64, P  # noqa: F401

pytestmark = pytest.mark.gpu


def chunk_width(M, V):
    """Columns of a chunk: of two copies of dz, rows and columns padded to 128, each within 2.5 GiB; even, of 256s."""
    rows, cols = (M + 127) // 128 * 128, (V + 127) // 128 * 128
    most = (5 << 29) // (2 * rows) // 256 * 256
    chunks = -(-cols // most)
    return chunks, min((-(-cols // chunks) + 255) // 256 * 256, cols)


@pytest.mark.parametrize("M,V,chunks,width", [(16384, 90001, 2, 45056), (30001, 131072, 3, 43776)])
def test_borders_of_chunks(P, M, V, chunks, width):  # noqa: F811
    import torch
    assert chunk_width(M, V) == (chunks, width)
    K, k = 16, 4
    c = Case(M + 1, M, V, K, k, plain=True)
    borders = [b for b in range(width, V, width)]
    near = np.array([b + d for b in borders for d in (-1, 0)] + [0, V - 1])
    marked = np.arange(5, M, 97)                               # rows with an entry at a border, some with one on both sides
    c.ids[marked, 0] = near[np.arange(marked.size) % near.size]
    c.ids[marked[::3], 2] = near[(np.arange(marked[::3].size) + 1) % near.size]
    c.dev = c.dev[:2] + (to_dev(c.ids), c.dev[3])
    lse, loss, z_top = P.lm_head_distill_fwd(*c.dev)
    dX, dW = P.lm_head_distill_bwd(*c.dev, lse, z_top, dloss=to_dev(c.dloss))
    rows = np.unique(np.r_[0, M - 1, marked[:24]])
    f = ld.forward(c.X[rows], c.W, c.ids[rows], c.t[rows], 1.0, L)
    for name, got in (("lse", lse), ("loss", loss)):
        assert (np.abs(host(got)[rows] - f[name]) <= f["tol_" + name] + 2.0 ** -24 * np.abs(f[name])).all(), name
    part = Case(0, 1, 1, 8, 1)
    part.X, part.W = c.X[rows], c.W
    check_gradients(part, f, 1.0, c.dloss[rows].astype(np.float64), 1.0, dX[torch.from_numpy(rows).cuda()], None)
    # dW's rows around the borders: those columns as a vocabulary, with the whole one's lse (checked above); entries
    # elsewhere count for Q and stand in a column of their own, dropped afterwards
    cols = np.unique(np.clip([b + d for b in borders for d in range(-3, 3)] + [0, V - 2, V - 1], 0, V - 1))
    x, w = f64(c.X), f64(c.W[cols])
    place = np.full(V, cols.size, np.int64)
    place[cols] = np.arange(cols.size)
    q, _, tol_q = ld.teacher(c.ids, c.t, V, 1.0, L)
    more = np.zeros((M, 1))
    g = dict(a=np.concatenate((x @ w.T, more), 1), tol_a=np.concatenate((ld.TOL_Z * (np.abs(x) @ np.abs(w).T), more), 1),
             lse=host(lse).astype(np.float64), tol_lse=np.zeros(M), q=q, tol_q=tol_q, at=place[c.ids])
    g["ok"] = np.ones_like(g["at"], bool)
    mid, lo, hi = (f64(v)[:, :-1] for v in ld.dz_band(g, 1.0, c.dloss.astype(np.float64), 1.0))
    check_fp32(host(dW[torch.from_numpy(cols).cuda()]), mid.T @ x, np.abs(mid).T @ np.abs(x), what="dW at the borders",
               slack=(hi - lo).T @ np.abs(x))


@pytest.mark.parametrize("M,V", [(300, 33001), (500, 32768), (257, 40003)])
def test_long_reduction_in_narrow_tiles(P, M, V):  # noqa: F811
    """Sizes of dX that leave fewer compute units idle in 256 x 192 tiles than in 256 x 256 ones, whole units and not."""
    K = 1536
    units = lambda n: 256 // (-(-M // 256) * -(-K // n)) * (-(-M // 256) * -(-K // n))
    assert 2 * ((V + 127) // 128 * 128) >= 65536 and units(192) > units(256)
    c = Case(M, M, V, K, 8)
    f, lse, loss, z_top = check_forward(P, c, 1.0)
    dX, _ = P.lm_head_distill_bwd(*c.dev, lse, z_top, dloss=to_dev(c.dloss), want_dw=False)
    check_gradients(c, f, 1.0, c.dloss.astype(np.float64), 1.0, dX, None)
