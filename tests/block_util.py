"""Matrices for the tests of layer norm and the gated block: numpy values beside a device matrix whose row padding holds NaN (inputs) or a
pattern that has to be found untouched (outputs), and the derived bounds that results are held to.

Bounds.  A bf16 result is the fp32 value rounded once: half a step, at most 2^-8 of it (BF16).  A sum of n products in fp32 is off by at
most about n 2^-24 of the sum of their magnitudes in any order (FP32 n); matrix instructions may drop bits where they align the products of a group,
for which the bound is doubled."""
import numpy as np
import torch

import paper_2305_13525_amd as axo

BF16 = 2.0 ** -8
FP32 = 2.0 ** -24
DEV = "cuda:0"


def problem(T, K, N, grid=(1, 1, 1), coord=(0, 0, 0), transposed=0):
    return axo.Problem.make(grid, coord, T, K, N, transposed)


def stream():
    return torch.cuda.current_stream().cuda_stream


def draw(rng, rows, cols, sigma=1.0, mean=0.0, wide=False):
    """float64 values that bf16 (or fp32) holds exactly."""
    a = torch.from_numpy((rng.standard_normal((rows, cols)) * sigma + mean).astype(np.float32))
    return (a if wide else a.bfloat16()).double().numpy()


class Mat:
    """A rows x cols matrix on the device with `gap` elements of padding behind rows rounded up to 8, which holds NaN; the last row has none."""

    def __init__(self, values, gap=0, wide=False):
        rows, cols = values.shape
        self.ld = (cols + 7) // 8 * 8 + gap
        self.rows, self.cols = rows, cols
        dtype = torch.float32 if wide else torch.bfloat16
        # the buffer ends with the matrix's last element, rounded up to the 16 bytes that allocations are made of anyway
        self.flat = torch.full((max(rows * self.ld, 8),), float("nan"), dtype=dtype, device=DEV)
        if rows and cols:
            self.view().copy_(torch.from_numpy(values).to(dtype))
        self.ptr = self.flat.data_ptr()

    def view(self):
        return self.flat.as_strided((self.rows, self.cols), (self.ld, 1))

    def numpy(self):
        return self.view().double().cpu().numpy()


class Out(Mat):
    """An output: NaN everywhere, so that what is not written shows."""

    def __init__(self, rows, cols, gap=0, wide=False):
        super().__init__(np.full((rows, cols), np.nan), gap, wide)

    def result(self):
        assert self.padding_untouched()
        return self.numpy()

    def padding_untouched(self):
        if self.rows == 0:
            return True
        pad = self.flat[:self.rows * self.ld].view(self.rows, self.ld)[:, self.cols:]
        return bool(torch.isnan(pad).all())


def vec(values, dtype=torch.bfloat16):
    return None if values is None else torch.from_numpy(np.ascontiguousarray(values)).to(dtype).to(DEV)


def ptr(t):
    return None if t is None else (t.ptr if isinstance(t, Mat) else t.data_ptr())


def within(got, want, bound, what=""):
    """|got - want| <= bound, element by element; `bound` an array or a number."""
    assert got.shape == want.shape, (what, got.shape, want.shape)
    if want.size == 0:
        return
    off = np.abs(got - want)
    assert np.all(np.isfinite(got)), (what, "not finite", np.argwhere(~np.isfinite(got))[:4])
    worst = np.unravel_index(np.argmax(off - bound), off.shape)
    assert np.all(off <= bound), (what, worst, got[worst], want[worst], float(off[worst]), float(np.broadcast_to(bound, off.shape)[worst]))


# bounds of the values that the kernels compute, all in terms of 64-bit quantities

def norm_bounds(s, mean, rstd, gamma, beta, y, wide):
    """Bound of y (bf16), of mean, of rstd (fp32)."""
    k = s.shape[1]
    eps_mean = (k * FP32 * np.abs(s).mean(axis=1) + FP32 * np.abs(mean))[:, None]   # of the mean
    dev = np.abs(s - mean[:, None])
    # rstd: half the relative error of the variance, sums of k squares of deviations each off by eps_mean and a rounding or two
    rel_rstd = (k + 8) * FP32 + (eps_mean[:, 0] * rstd) ** 2
    bound_h = (dev * (rel_rstd[:, None] + 4 * FP32) + eps_mean) * rstd[:, None]
    scale = 1.0 if gamma is None else np.abs(gamma)
    bound_y = BF16 * np.abs(y) + 2 * bound_h * scale + 4 * FP32 * (dev * rstd[:, None] * scale + (0 if beta is None else np.abs(beta)))
    return bound_y + 1e-38, eps_mean[:, 0] + 1e-38, (rel_rstd + 4 * FP32) * rstd


def norm_bwd_bounds(dy, s, mean, rstd, gamma, r, dx, wide):
    """Bounds of dx, dgamma, dbeta."""
    m, k = s.shape
    h = (s - mean[:, None]) * rstd[:, None]
    err_h = FP32 * (np.abs(s) + np.abs(mean)[:, None]) * rstd[:, None] * 2 + 2 * FP32 * np.abs(h)
    g = np.abs(dy if gamma is None else dy * gamma)
    c1 = (k + 4) * FP32 * g.mean(axis=1)[:, None]
    c2 = ((k + 4) * FP32 * (g * np.abs(h)).mean(axis=1) + (g * err_h).mean(axis=1))[:, None]
    inner = c1 + np.abs(h) * c2 + err_h * (g * np.abs(h)).mean(axis=1)[:, None] + 8 * FP32 * (g + g.mean(axis=1)[:, None] + np.abs(h) * (g * np.abs(h)).mean(axis=1)[:, None])
    bound = rstd[:, None] * inner + (0 if r is None else 2 * FP32 * np.abs(r)) + (2 * FP32 if wide else BF16) * np.abs(dx)
    dg = (m + 8) * FP32 * (np.abs(dy) * np.abs(h)).sum(axis=0) + (np.abs(dy) * err_h).sum(axis=0)
    db = (m + 8) * FP32 * np.abs(dy).sum(axis=0)
    return bound + 1e-38, dg + 1e-30, db + 1e-30


def product_bound(a, b):
    """Of an fp32 sum a @ b."""
    return 2 * (a.shape[1] + 4) * FP32 * (np.abs(a) @ np.abs(b))


# of an activation's value or derivative in fp32, relative to max(1, |v|): exp2 of an argument off by up to 128 * 2^-24, reciprocal, polynomials;
# 3e-6 of the value at the far ends, 1e-6 elsewhere
ACT = 4e-6
SLOPE = 1.13  # largest |act'| of the three


def gated_fwd_bounds(x, wg, wu, g, u, value, bg=None, bu=None):
    """Bounds of h, g, u."""
    eg = product_bound(x, wg) + FP32 * np.abs(g) * 2
    eu = product_bound(x, wu) + FP32 * np.abs(u) * 2
    h = np.abs(value * u)
    bound_h = BF16 * h + np.abs(u) * (SLOPE * eg + ACT * np.maximum(1.0, np.abs(g))) + np.abs(value) * eu + SLOPE * eg * eu
    return bound_h + 1e-38, BF16 * np.abs(g) + eg + 1e-38, BF16 * np.abs(u) + eu + 1e-38


def gated_dact_bounds(err_dh, dh, g, u, value, slope):
    """Bounds of dg, du where dh is off by err_dh."""
    act = ACT * np.maximum(1.0, np.abs(g))
    dg = BF16 * np.abs(dh * u * slope) + np.abs(u) * (err_dh * (np.abs(slope) + act) + np.abs(dh) * act) + 4 * FP32 * np.abs(dh * u * slope)
    du = BF16 * np.abs(dh * value) + err_dh * (np.abs(value) + act) + np.abs(dh) * act + 4 * FP32 * np.abs(dh * value)
    return dg + 1e-38, du + 1e-38
