"""The orthogonalised update with X, A and Q rounded where the kernels round them, and how far O may be off its definition."""
import numpy as np
import torch

import block_util as bu
import residual_util as ru
from oracle import residual as orr

BF, HALF = torch.bfloat16, torch.float16


def to(dtype, a):
    return torch.from_numpy(a).to(dtype).double().numpy()


def update(g, held, steps=5, eps=0.0):
    """The iterate in 64 bits but for X, times a power of two, A and Q, which are held in `held`; O not rounded."""
    tall = g.shape[0] > g.shape[1]
    x = g.T if tall else g
    scale = 2.0 ** min(13, int(0.5 * np.log2(g.size)))
    x = to(held, x * (scale / (np.linalg.norm(x) + eps)))
    a, b, c = orr.QUINTIC
    for i in range(steps):
        m = to(held, x @ x.T / scale ** 2)
        x = to(held, a * np.eye(len(m)) + b * m + c * (m @ m)) @ x
        if i + 1 < steps:
            x = to(held, x)
    return (x.T if tall else x) / scale


# k, n; how singular values lie; what is documented of |O - exact| / |exact| ahead of O's rounding
RANDOM, HUNDRED = 0.002, 0.005
SIZES = [(40, 40), (64, 130), (130, 70), (200, 200), (128, 512), (515, 259), (257, 1000), (64, 4096), (1000, 1030), (640, 2500), (60, 5000), (3000, 72)]
CASES = [(k, n, None, RANDOM) for k, n in SIZES] + [(k, n, 100.0, HUNDRED) for k, n in SIZES]


def gradient(k, n, spread):
    """fp32 values: a random matrix, or one with its singular vectors whose singular values lie evenly, in their logarithm, over a factor of `spread`."""
    g = bu.draw(np.random.default_rng(k + 3 * n), k, n, 1e-3, 0.0, True)
    if spread is None:
        return g
    u, _, v = np.linalg.svd(g, full_matrices=False)
    return to(torch.float32, (u * np.geomspace(1.0, 1.0 / spread, min(k, n))) @ v)


def check(got, want, documented):
    """The update as a whole: what is documented, and the rounding to bf16, which takes from `got` what it takes from `want`, statistically: over 1600 values and more their norms are
    alike within a tenth.  Each row and column: twice its share of the former, and half a step of bf16."""
    assert np.isfinite(got).all()
    size, rounding = np.linalg.norm(want), np.linalg.norm(to(BF, want) - want)
    off = np.linalg.norm(got - want)
    assert off <= documented * size + 1.1 * rounding, (off / size, rounding / size)
    for axis in (0, 1):
        share = size / np.sqrt(want.shape[1 - axis])
        over = np.linalg.norm(got - want, axis=axis) - ru.BF16 * np.linalg.norm(want, axis=axis)
        assert over.max() <= 2 * documented * share, (axis, over.max() / share)
