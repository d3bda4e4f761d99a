"""Bounds of the residual addition's operators and of the orthogonalised update, all in terms of 64-bit quantities; BF16, FP32 and the bounds of sums and activations are
those of block_util."""
import numpy as np

import block_util as bu
from oracle import residual as orr

BF16, FP32 = bu.BF16, bu.FP32
FP16 = 2.0 ** -11


def fc_add_bounds(x, w, r, z, y, scale, epilogue, wide):
    """Bounds of y and of z.  The activation's slope is at most SLOPE, its own error ACT of max(1, |z|)."""
    ez = bu.product_bound(x, w) + 2 * FP32 * np.abs(z)
    inner = bu.SLOPE * ez + bu.ACT * np.maximum(1.0, np.abs(z)) if epilogue >= 2 else ez
    value = np.abs(scale * orr.act(z, epilogue)[0])
    bound = np.abs(scale) * inner + 2 * FP32 * (value + (0 if r is None else np.abs(r))) + (FP32 if wide else BF16) * np.abs(y)
    return bound + 1e-38, BF16 * np.abs(z) + ez + 1e-38


def dact_bound(dy, z, scale, epilogue, dz):
    return BF16 * np.abs(dz) + 4 * FP32 * np.abs(dz) + (0 if epilogue < 2 else np.abs(scale * dy) * bu.ACT * np.maximum(1.0, np.abs(z))) + 1e-38


def normed_bounds(v, kind, mean, rstd):
    """Errors of a row's mean, of its rstd and of its normed values in fp32."""
    k = v.shape[1]
    if kind == orr.NONE:
        return np.zeros(len(v)), np.zeros(len(v)), np.zeros_like(v)
    em = k * FP32 * np.abs(v).mean(axis=1) + FP32 * np.abs(mean) if kind == orr.LAYER else np.zeros(len(v))
    dev = np.abs(v - mean[:, None])
    rel = (k + 8) * FP32 + (em * rstd) ** 2
    return em, (rel + 4 * FP32) * rstd, (dev * (rel[:, None] + 4 * FP32) + em[:, None]) * rstd[:, None]


def s_bound(b, x, scale, kind, mean, rstd, gamma, beta, gate, s, wide):
    *_, eh = normed_bounds(b, kind, mean, rstd)
    h = np.abs(orr.normed(b, mean, rstd))
    ez = eh * np.abs(gamma) + 4 * FP32 * (h * np.abs(gamma) + np.abs(beta))
    z = h * np.abs(gamma) + np.abs(beta)
    return np.abs(scale * gate) * (ez + 4 * FP32 * z) + 2 * FP32 * np.abs(x) + (FP32 if wide else BF16) * np.abs(s) + 1e-38


def y_bound(s, kind, mean, rstd, gamma, beta, y):
    *_, eh = normed_bounds(s, kind, mean, rstd)
    return BF16 * np.abs(y) + 2 * eh * np.abs(gamma) + 4 * FP32 * (np.abs(orr.normed(s, mean, rstd) * gamma) + np.abs(beta)) + 1e-38


def _back_bound(g, eg, h, eh, rstd, kind, k):
    """Of norm_back in fp32, g off by eg and h by eh."""
    if kind == orr.NONE:
        return eg
    mean = lambda v: v.mean(axis=1)[:, None]  # noqa: E731
    g, h = np.abs(g), np.abs(h)
    inner = eg + h * (mean(eg * h + g * eh) + (k + 4) * FP32 * mean(g * h)) + eh * mean(g * h) + 8 * FP32 * (g + h * mean(g * h))
    if kind == orr.LAYER:
        inner = inner + mean(eg) + (k + 12) * FP32 * mean(g)
    return rstd[:, None] * inner


def resnorm_bwd_bounds(dy, ds, b, s, stats, scale, kind_a, kind_b, gamma_a, beta_a, gate, gamma_b, want, wide):
    """Bounds of what orr.resnorm_bwd returns."""
    m, k = dy.shape
    normed_error = lambda v, mean, rstd, h: 2 * FP32 * (np.abs(v) + np.abs(mean)[:, None]) * rstd[:, None] + 2 * FP32 * np.abs(h)  # noqa: E731
    ha, hb = orr.normed(b, stats[:, 0], stats[:, 1]), orr.normed(s, stats[:, 2], stats[:, 3])
    ea, eb = normed_error(b, stats[:, 0], stats[:, 1], ha), normed_error(s, stats[:, 2], stats[:, 3], hb)
    dx, db = want[0], want[1]
    e_ds = _back_bound(dy * gamma_b, 2 * FP32 * np.abs(dy * gamma_b), hb, eb, stats[:, 3], kind_b, k) + 2 * FP32 * np.abs(dx) + (0 if ds is None else 2 * FP32 * np.abs(ds))
    q = np.abs(scale * gate * gamma_a)
    e_q = q * (e_ds + 4 * FP32 * np.abs(dx))
    e_db = _back_bound(q * dx, e_q, ha, ea, stats[:, 1], kind_a, k)
    total = lambda v, e: (m + 8) * FP32 * np.abs(v).sum(axis=0) + e.sum(axis=0)  # noqa: E731
    b0, b1 = total(dx * ha, e_ds * np.abs(ha) + np.abs(dx) * ea), total(dx, e_ds)
    s0, s1 = np.abs((dx * ha).sum(axis=0)), np.abs(dx.sum(axis=0))
    g = np.abs(scale * gate)
    return (e_ds + (2 * FP32 if wide else BF16) * np.abs(dx) + 1e-38, e_db + BF16 * np.abs(db) + 1e-38, g * (b0 + 4 * FP32 * s0) + 1e-30, g * (b1 + 4 * FP32 * s1) + 1e-30,
            np.abs(scale) * (np.abs(gamma_a) * (b0 + 8 * FP32 * s0) + np.abs(beta_a) * (b1 + 8 * FP32 * s1)) + 1e-30,
            total(dy * hb, np.abs(dy) * eb) + 1e-30, total(dy, 0 * dy) + 1e-30)


def ortho_bound(g, steps, abc=None, eps=0.0):
    """Bound of |O - exact| in the Frobenius norm.  A step that starts off by E ends off by at most L E, L the largest slope between any two of the singular values involved
    (and between one and another's negative, the polynomial being odd), and adds what it rounds: X to fp16, A to fp16, Q to fp16, each by FP16 of its values.  To first order,
    with an eighth more for the others; fp32 sums are off by less than an eighth of these again."""
    path = []
    want = orr.ortho(g, steps, abc, eps, path)
    off = FP16 * np.linalg.norm(path[0])
    for i, x in enumerate(path):
        a, b, c = orr.QUINTIC if abc is None else abc[3 * i:3 * i + 3]
        v = np.linalg.svd(x, compute_uv=False)
        top = v.max()
        poly = lambda t: a * t + b * t ** 3 + c * t ** 5  # noqa: E731, B023
        t = np.concatenate([-v, v])
        t, p = t[:, None], poly(t)[:, None]
        gap = t - t.T
        slope = np.abs(np.divide(p - p.T, gap, out=np.zeros_like(gap), where=np.abs(gap) > 1e-9 * top)).max()
        slope = max(slope, np.abs(a + 3 * b * v ** 2 + 5 * c * v ** 4).max())
        gram = v ** 2
        q = a + b * gram + c * gram ** 2
        from_gram = (abs(b) + 2 * abs(c) * top ** 2) * FP16 * np.linalg.norm(gram) * top
        from_q = FP16 * np.sqrt((q ** 2).sum()) * top
        after = FP16 * np.linalg.norm(poly(v)) if i + 1 < steps else 0.0
        off = slope * off + from_gram + from_q + after
    return want, 1.25 * off + BF16 * np.linalg.norm(want)
