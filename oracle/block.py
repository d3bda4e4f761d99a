"""Layer norm and the gated feed-forward block in 64 bits, from their definitions (plain numpy; arrays of float64 in, float64 out)."""
import math

import numpy as np

_erf = np.frompyfunc(math.erf, 1, 1)
SILU, GELU_TANH, GELU_ERF = 0, 1, 2


def norm_fwd(s, gamma=None, beta=None, eps=1e-5):
    """(y, mean, rstd) of each row."""
    mean = s.mean(axis=1)
    rstd = 1.0 / np.sqrt(((s - mean[:, None]) ** 2).mean(axis=1) + eps)
    y = (s - mean[:, None]) * rstd[:, None]
    if gamma is not None:
        y = y * gamma
    if beta is not None:
        y = y + beta
    return y, mean, rstd


def norm_bwd(dy, s, mean, rstd, gamma=None, r=None):
    """(dx, dgamma, dbeta), the statistics given."""
    h = (s - mean[:, None]) * rstd[:, None]
    g = dy if gamma is None else dy * gamma
    dx = rstd[:, None] * (g - g.mean(axis=1)[:, None] - h * (g * h).mean(axis=1)[:, None])
    return dx if r is None else dx + r, (dy * h).sum(axis=0), dy.sum(axis=0)


def gate(v, kind):
    """(act(v), act'(v))"""
    if kind == SILU:
        p = 1.0 / (1.0 + np.exp(-v))
        return v * p, p + v * p * (1.0 - p)
    if kind == GELU_TANH:
        c = math.sqrt(2.0 / math.pi)
        t = np.tanh(c * (v + 0.044715 * v ** 3))
        return 0.5 * v * (1.0 + t), 0.5 * (1.0 + t) + 0.5 * v * (1.0 - t * t) * c * (1.0 + 3.0 * 0.044715 * v * v)
    p = 0.5 * (1.0 + _erf(v / math.sqrt(2.0)).astype(np.float64))
    return v * p, p + v * np.exp(-0.5 * v * v) / math.sqrt(2.0 * math.pi)


def gated_fwd(x, wg, wu, kind, bg=None, bu=None):
    """(h, g, u)"""
    g, u = x @ wg, x @ wu
    if bg is not None:
        g = g + bg
    if bu is not None:
        u = u + bu
    return gate(g, kind)[0] * u, g, u


def gated_dact(dh, g, u, kind):
    """(dg, du)"""
    value, slope = gate(g, kind)
    return dh * u * slope, dh * value


def gated_dgrad(dg, du, wg, wu):
    return dg @ wg.T + du @ wu.T
