"""The example that runs layer norm, the gated block and the fully-connected layer together: it learns, its gradients are those of the whole
sublayer, and a token on its own gets the answer that it gets in a batch."""
import os
import sys

import numpy as np
import pytest

torch = pytest.importorskip("torch")
import block_util as bu
from oracle import block as ob

sys.path.insert(0, os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples"))
gated_mlp = pytest.importorskip("gated_mlp")
pytestmark = pytest.mark.gpu


def test_it_learns():
    losses, apart = gated_mlp.main(["--tokens", "512", "--width", "256", "--inner", "704", "--steps", "12"])
    assert all(b < a for a, b in zip(losses, losses[1:])) and losses[-1] < 0.9 * losses[0]
    # the two answers are sums in another order, each rounded to bf16 several times on the way: a few steps of values below 8
    assert apart <= 4 * bu.BF16 * 8


@pytest.mark.parametrize("tokens", [1, 40, 300])
def test_gradients_of_the_sublayer(tokens):
    """Against the 64-bit definition on the same bf16 weights.  Every tensor between the calls is rounded to bf16 (n, G, U, H, dG, dU, dn): some seven roundings of
    2^-9 rms each stand behind a gradient, which is 1 % where their errors add up unfavourably in the 2-norm."""
    width, inner = 96, 160
    net = gated_mlp.GatedMLP(tokens, width, inner, seed=4)
    rng = np.random.default_rng(5)
    x, dy = bu.draw(rng, tokens, width), bu.draw(rng, tokens, width)
    net.w["gamma"].copy_(bu.vec(1 + bu.draw(rng, 1, width, 0.1)[0]))
    net.w["beta"].copy_(bu.vec(bu.draw(rng, 1, width, 0.1)[0]))
    for k in ("wg", "wu", "wd"):
        net.w[k].mul_(8.0)
    X, DY = bu.vec(x), bu.vec(dy)
    y = net.forward(X)
    dx = net.backward(X, DY)
    w = {k: v.double().cpu().numpy() for k, v in net.w.items()}
    n, mean, rstd = ob.norm_fwd(x, w["gamma"], w["beta"], gated_mlp.EPS)
    h, g, u = ob.gated_fwd(n, w["wg"], w["wu"], 0)
    dg, du = ob.gated_dact(dy @ w["wd"].T, g, u, 0)
    dn = ob.gated_dgrad(dg, du, w["wg"], w["wu"])
    want = {"wd": h.T @ dy, "wg": n.T @ dg, "wu": n.T @ du}
    want_dx, want["gamma"], want["beta"] = ob.norm_bwd(dn, x, mean, rstd, w["gamma"], dy)
    off = lambda a, b: np.linalg.norm(a - b) / np.linalg.norm(b)  # noqa: E731
    back = lambda t: t.double().cpu().numpy()  # noqa: E731
    assert off(back(y), x + h @ w["wd"]) <= 0.01
    assert off(back(dx), want_dx) <= 0.01
    for k, v in want.items():
        assert off(back(net.grad[k]), v) <= 0.01, k


def test_fewer_tokens_than_there_are_buffers_for():
    """The same bits as from a sublayer of that size, and gradients of as many rows as there are tokens."""
    rng = np.random.default_rng(6)
    x, dy = bu.vec(bu.draw(rng, 40, 96)), bu.vec(bu.draw(rng, 40, 96))
    got = []
    for tokens in (300, 40):
        net = gated_mlp.GatedMLP(tokens, 96, 160, seed=4)
        got.append((net.forward(x), net.backward(x, dy).clone(), net.grad))
    (y, dx, grad), (y2, dx2, grad2) = got
    assert dx.shape == x.shape and torch.equal(y, y2) and torch.equal(dx, dx2)
    assert all(torch.equal(grad[k], grad2[k]) for k in grad)
    with pytest.raises(ValueError):
        gated_mlp.GatedMLP(39, 96, 160).forward(x)
