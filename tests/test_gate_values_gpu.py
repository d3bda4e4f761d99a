"""The gate's activations and their derivatives value by value, through the element-wise calls, each result held to its own size: far below zero an
activation is small, not zero, down to the smallest normal numbers."""
import math

import numpy as np
import pytest

torch = pytest.importorskip("torch")
import block_util as bu
import paper_2305_13525_amd as axo

SILU, TANH, ERF = axo.AXO_GATE_SILU, axo.AXO_GATE_GELU_TANH, axo.AXO_GATE_GELU_ERF

# Relative error of the arithmetic, ahead of the rounding to bf16: that of exp2's argument, which passes 126 (erf: 190) in magnitude, times ln 2.  SiLU: the constant and one
# product, 1.5 * 2^-24 each of 126, 8e-6; tanh form: two constants, v^2, a fused and a plain product, 4 * 2^-24 of 126, 2.1e-5; erf form: the same of one constant
# and two roundings of 190, 2.4e-5, and the polynomial's 2e-6.  exp2, reciprocal and the products around them a few 2^-24 more.
RELATIVE = 4e-5
LOST = 2.0 ** -126  # neither exp2 nor the reciprocal has results below: a sigmoid or a Gaussian, and what it is multiplied with, may be zero there


def values():
    """All finite bf16 numbers below 2^120 in magnitude."""
    with np.errstate(invalid="ignore"):
        g = (np.arange(1 << 16, dtype=np.uint32) << 16).view(np.float32).astype(np.float64)
    return np.sort(g[np.isfinite(g) & (np.abs(g) < 2.0 ** 120)])


def forms(v, kind):
    """(value, bound of its error), (slope, bound), where there may be zeros instead: the 64-bit forms without cancellation below zero."""
    with np.errstate(over="ignore", invalid="ignore"):
        if kind == ERF:
            x = np.clip(v, -40.0, 40.0)
            p = np.array([0.5 * math.erfc(-t / math.sqrt(2.0)) for t in x])
            change = np.exp(-0.5 * x * x) / math.sqrt(2.0 * math.pi)  # p'
        elif kind == TANH:
            x, c = np.clip(v, -40.0, 40.0), math.sqrt(8.0 / math.pi)
            p, q = (1.0 / (1.0 + np.exp(t * c * (x + 0.044715 * x ** 3))) for t in (-1.0, 1.0))
            change = p * q * c * (1.0 + 3.0 * 0.044715 * x * x)
        else:
            x = np.clip(v, -700.0, 700.0)
            p, q = 1.0 / (1.0 + np.exp(-x)), 1.0 / (1.0 + np.exp(x))
            change = p * q
        value = np.where(v > x, v, x * p)
        slope = p + x * change
        size = p + np.abs(x) * change  # of the terms that the slope is the sum of
    lost = (v < 0.0) & ((np.exp(-0.5 * x * x) if kind == ERF else p) < 2.0 * LOST)
    half_step = 2.0 ** -134  # of bf16's subnormal numbers
    bound_value = (bu.BF16 + RELATIVE) * np.abs(value) + np.where(lost & (kind != ERF), np.abs(value), 0.0) + half_step
    bound_slope = bu.BF16 * np.abs(slope) + RELATIVE * size + np.where(lost, size, 0.0) + half_step
    return (value, bound_value), (slope, bound_slope), lost


@pytest.mark.parametrize("kind", [SILU, TANH, ERF])
def test_bounds_tell(kind):
    """Nothing but a rounding is allowed as far down as the arithmetic's range goes, and for slopes not next to their zero: to -87 (SiLU), -9.9 (tanh form), -13 (erf form)."""
    v = values()
    (value, bound_value), (slope, bound_slope), lost = forms(v, kind)
    assert v[~lost].min() <= {SILU: -86.5, TANH: -9.9375, ERF: -13.0}[kind] and not lost[v > {SILU: -86.5, TANH: -9.9375, ERF: -13.0}[kind]].any()
    there = (np.abs(value) > 2.0 ** -126) & (~lost | (kind == ERF))
    assert np.all(bound_value[there] < 0.01 * np.abs(value[there]))
    there = (v < -4.0) & ~lost
    assert np.all(bound_slope[there] < 0.01 * np.abs(slope[there]))


@pytest.mark.gpu
@pytest.mark.parametrize("kind", [SILU, TANH, ERF])
def test_every_value(kind):
    v = values()
    g = v[:v.size // 8 * 8].reshape(-1, 8)
    one = np.ones_like(g)
    G, U, H, dG, dU = bu.Mat(g), bu.Mat(one), bu.Out(*g.shape), bu.Out(*g.shape), bu.Out(*g.shape)
    p = bu.problem(g.shape[0], 8, 8)
    axo.axo_gated_act(p, G.ptr, U.ptr, G.ld, kind, H.ptr, H.ld, bu.stream())
    axo.axo_gated_dact(p, U.ptr, U.ld, G.ptr, U.ptr, G.ld, kind, dG.ptr, dU.ptr, dG.ld, bu.stream())
    (value, bound_value), (slope, bound_slope), _ = forms(g.ravel(), kind)
    bu.within(H.result().ravel(), value, bound_value, "value")
    assert np.array_equal(H.result(), dU.result())
    bu.within(dG.result().ravel(), slope, bound_slope, "slope")


@pytest.mark.gpu
@pytest.mark.parametrize("kind", [SILU, TANH, ERF])
def test_the_same_in_the_products(kind):
    """A reduction of one term: the epilogues' values and those of the derivative's are the element-wise ones, bit for bit."""
    v = values()
    g = np.resize(v, (-(-v.size // 64), 64))
    m = g.shape[0]
    # forward: G = v * 1, U = 1, a column of v at a time
    col = v.reshape(-1, 1)
    X = bu.Mat(np.concatenate([col, np.ones_like(col)], 1))
    Wg, Wu = bu.Mat(np.array([[1.0] * 8, [0.0] * 8])), bu.Mat(np.array([[0.0] * 8, [1.0] * 8]))
    H, E = bu.Out(col.size, 8), bu.Out(col.size, 8)
    p = bu.problem(col.size, 2, 8)
    n = axo.axo_gated_workspace_bytes(p)
    ws = torch.zeros(max(n, 16), dtype=torch.uint8, device=bu.DEV)
    axo.axo_gated_fwd(p, X.ptr, X.ld, Wg.ptr, Wu.ptr, Wg.ld, None, None, kind, None, None, 0, H.ptr, H.ld, ws.data_ptr(), n, bu.stream())
    G, U = bu.Mat(np.repeat(col, 8, 1)), bu.Mat(np.ones((col.size, 8)))
    axo.axo_gated_act(bu.problem(col.size, 8, 8), G.ptr, U.ptr, G.ld, kind, E.ptr, E.ld, bu.stream())
    assert np.array_equal(H.result(), E.result())
    # through the activation: dH = 1 * 1
    dY, W, G, U = bu.Mat(np.ones((m, 1))), bu.Mat(np.ones((64, 1))), bu.Mat(g), bu.Mat(np.ones_like(g))
    one, outs = bu.Mat(np.ones_like(g)), [bu.Out(m, 64) for _ in range(4)]
    p = bu.problem(m, 64, 1)
    n = axo.axo_gated_workspace_bytes(p)
    ws = torch.zeros(max(n, 16), dtype=torch.uint8, device=bu.DEV)
    axo.axo_gated_dgrad_act(p, dY.ptr, dY.ld, W.ptr, W.ld, G.ptr, U.ptr, G.ld, kind, outs[0].ptr, outs[1].ptr, outs[0].ld, ws.data_ptr(), n, bu.stream())
    axo.axo_gated_dact(p, one.ptr, one.ld, G.ptr, U.ptr, G.ld, kind, outs[2].ptr, outs[3].ptr, outs[2].ld, bu.stream())
    assert np.array_equal(outs[0].result(), outs[2].result()) and np.array_equal(outs[1].result(), outs[3].result())
