"""The int8 oracle's band of the fused RMSNorm against the additions that the sum of
squares goes through on its way."""

import numpy as np
import pytest

from oracle import int8

U = 2.0 ** -24


def layout(R, C):
    """Threads of a row: a row's chunks of 8 values lie on them in turn."""
    if R >= 4096 and C <= 128:
        return 16
    return 64 if R >= 1024 and C <= 2048 else 256


def roundings(R, C):
    """Roundings between a square and the sum of its row: of the lanes' chains, over the lanes of a wave, over four waves."""
    threads, chunks = layout(R, C), C // 8
    chain = [8 * len(range(t, chunks, threads)) for t in range(threads)]
    depth = []
    for w in range(0, threads, 64):
        d = chain[w:w + 64]
        o = len(d) // 2
        while o >= 1:
            d = [max(d[i], d[i ^ o]) + 1 for i in range(len(d))]
            o //= 2
        depth.append(d[0])
    if len(depth) == 4:
        depth = [max(max(depth[0], depth[1]), max(depth[2], depth[3])) + 2]
    return depth[0]


SHAPES = [(1, 16), (3, 48), (33, 2048), (1, 2056), (5, 17920), (2, 65552), (1023, 1536), (1024, 1536), (2500, 528), (4095, 128),
          (4096, 128), (4096, 136), (5000, 2048), (5000, 2064)]


@pytest.mark.parametrize("R,C", SHAPES)
def test_allowance_covers_every_rounding(R, C):
    x = np.ones((R, C))
    # (halved by the root; the mean's division, eps, root, reciprocal and two products)
    assert int8.rmsnorm(x, np.ones(C), 1e-6)[2] >= (roundings(R, C) / 2 + 6) * U


@pytest.mark.parametrize("R,C", [(1, 16), (3, 48), (1024, 528), (4096, 128), (2, 2064)])
def test_a_binary32_evaluation_is_inside(R, C):
    g = np.random.default_rng(C)
    x = (g.normal(size=(R, C)) * np.exp(g.normal(size=(R, 1)))).astype(np.float32)
    x = (x.view(np.uint32) & 0xFFFF0000).view(np.float32)
    gamma = np.ones(C, np.float32)
    f, threads = np.float32, layout(R, C)
    lanes = np.zeros((R, threads), np.float32)
    for c in range(C // 8):
        for e in range(8):
            v = x[:, c * 8 + e].astype(np.float64)
            lanes[:, c % threads] = (v * v + lanes[:, c % threads]).astype(np.float32)       # (fused)
    waves = [lanes[:, w:w + 64] for w in range(0, threads, 64)]
    for i, w in enumerate(waves):
        o = w.shape[1] // 2
        while o >= 1:
            w = w + w[:, np.arange(w.shape[1]) ^ o]
            o //= 2
        waves[i] = w[:, 0]
    ss = waves[0] if len(waves) == 1 else (waves[0] + waves[1]) + (waves[2] + waves[3])
    rstd = f(1) / np.sqrt(ss / f(C) + f(1e-6))
    y = x * rstd[:, None] * gamma
    ref, want, e = int8.rmsnorm(x.astype(np.float64), gamma.astype(np.float64), float(f(1e-6)))
    assert (np.abs(rstd - want) <= e * want).all() and (np.abs(y - ref) <= e * np.abs(ref)).all()
