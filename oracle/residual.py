"""The residual addition's operators and the orthogonalised update in 64 bits, from their definitions (plain numpy; arrays of float64 in, float64 out)."""
import numpy as np

from . import block

NONE, LAYER, RMS = 0, 1, 2
QUINTIC = (3.4445, -4.7750, 2.0315)


def act(z, epilogue):
    """(act(z), act'(z)) of an axo_epilogue_t."""
    if epilogue < 2:
        return z, np.ones_like(z)
    return block.gate(z, block.GELU_TANH if epilogue == 2 else block.GELU_ERF)


def fc_add(x, w, r, scale, epilogue, bias=None):
    """(y, z)"""
    z = x @ w
    if bias is not None:
        z = z + bias
    y = scale * act(z, epilogue)[0]
    return y if r is None else r + y, z


def moments(v, kind, eps):
    """(mean, 1 / deviation) of each row."""
    m = len(v)
    if kind == NONE:
        return np.zeros(m), np.ones(m)
    mean = v.mean(axis=1) if kind == LAYER else np.zeros(m)
    return mean, 1.0 / np.sqrt(((v - mean[:, None]) ** 2).mean(axis=1) + eps)


def normed(v, mean, rstd):
    return (v - mean[:, None]) * rstd[:, None]


def resnorm_s(b, x, scale, kind, gamma=1.0, beta=0.0, gate=1.0, eps=1e-5):
    """(s, mean_a, rstd_a)"""
    mean, rstd = moments(b, kind, eps)
    return x + scale * gate * (normed(b, mean, rstd) * gamma + beta), mean, rstd


def resnorm_y(s, kind, gamma=1.0, beta=0.0, eps=1e-5):
    """(y, mean_b, rstd_b)"""
    mean, rstd = moments(s, kind, eps)
    return normed(s, mean, rstd) * gamma + beta, mean, rstd


def norm_back(g, h, rstd, kind):
    """The gradient of a norm's input from that of its normed rows h."""
    if kind == NONE:
        return g
    d = g - h * (g * h).mean(axis=1)[:, None]
    if kind == LAYER:
        d = d - g.mean(axis=1)[:, None]
    return d * rstd[:, None]


def resnorm_bwd(dy, ds, b, s, stats, scale, kind_a, kind_b, gamma_a=1.0, beta_a=0.0, gate=1.0, gamma_b=1.0):
    """(dx, db, dgamma_a, dbeta_a, dgate, dgamma_b, dbeta_b), the statistics given."""
    ha, hb = normed(b, stats[:, 0], stats[:, 1]), normed(s, stats[:, 2], stats[:, 3])
    dx = norm_back(dy * gamma_b, hb, stats[:, 3], kind_b)
    if ds is not None:
        dx = dx + ds
    dz = scale * gate * dx
    return (dx, norm_back(dz * gamma_a, ha, stats[:, 1], kind_a), (dz * ha).sum(axis=0), dz.sum(axis=0), (scale * dx * (ha * gamma_a + beta_a)).sum(axis=0),
            (dy * hb).sum(axis=0), dy.sum(axis=0))


def ortho(g, steps, abc=None, eps=0.0, path=None):
    """The Newton-Schulz iterate; `path`: a list that receives X of every step, on the side where X X^T is the smaller Gram matrix."""
    tall = g.shape[0] > g.shape[1]
    x = g.T if tall else g
    norm = np.sqrt((x ** 2).sum()) + eps
    x = x / norm if norm > 0 else x
    for i in range(steps):
        if path is not None:
            path.append(x)
        a, b, c = QUINTIC if abc is None else abc[3 * i:3 * i + 3]
        m = x @ x.T
        x = a * x + (b * m + c * (m @ m)) @ x
    return x.T if tall else x
