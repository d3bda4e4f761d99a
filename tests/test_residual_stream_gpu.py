"""The example that runs the norms around a residual addition, the product that adds to the residual stream and the orthogonalised update together with the gated block and the
fully-connected layer: its gradients are those of the whole stack, its updates those of the momenta, and a captured step does what the calls do one by one."""
import os
import sys

import numpy as np
import pytest

torch = pytest.importorskip("torch")
import block_util as bu
import residual_util as ru

sys.path.insert(0, os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples"))
residual_stream = pytest.importorskip("residual_stream")
pytestmark = pytest.mark.gpu


def test_it_runs():
    losses = residual_stream.main(["--tokens", "256", "--width", "128", "--inner", "192", "--layers", "3", "--steps", "3"])
    assert len(losses) == 3 and np.isfinite(losses).all()


def stack(tokens, layers, width=96, inner=160):
    """A stack whose vectors differ from ones and zeros, an input and a gradient."""
    net = residual_stream.Stream(tokens, width, inner, layers, seed=layers)
    rng = np.random.default_rng(tokens)
    for master, w in zip(net.master, net.w):
        for k in master:
            if master[k].dim() == 1:
                master[k].add_(bu.vec(bu.draw(rng, 1, width, 0.1)[0]).float())
                w[k].copy_(master[k])
    return net, *(torch.from_numpy(rng.standard_normal((tokens, width))).float().to(bu.DEV) for _ in range(2))


def plain(net, x):
    """The stack in 64 bits on the CPU: its output, and its weights as leaves."""
    w = [{k: v.double().cpu().requires_grad_() for k, v in layer.items()} for layer in net.w]
    x = x.double().cpu().requires_grad_()
    norm = lambda s, v: torch.nn.functional.layer_norm(s, s.shape[1:], v["gamma"], v["beta"], residual_stream.EPS)  # noqa: E731
    s = x
    for i, v in enumerate(w):
        n = norm(s, v)
        o = (torch.nn.functional.silu(n @ v["wg"]) * (n @ v["wu"])) @ v["wd"]
        if i + 1 == len(w):
            return s + net.scale * o, x, w
        s = s + v["gate"] * v["post"] * o / torch.sqrt(o.square().mean(dim=1, keepdim=True) + residual_stream.EPS)


@pytest.mark.parametrize("tokens,layers", [(1, 2), (40, 1), (300, 2), (130, 3)])
def test_gradients_of_the_stack(tokens, layers):
    """In 64 bits on the same bf16 weights.  A sublayer rounds seven tensors to bf16 on the way of a gradient (n, G or U, H, o; do, dG or dU, dn), each off by at most 2^-9 of its values'
    root mean square on average; these errors add up to at most their sum, as what they go through (normed rows, matrices of columns of length one, a gate) does not lengthen
    them on average."""
    net, x, dy = stack(tokens, layers)
    y, leaf, w = plain(net, x)
    y.backward(dy.double().cpu())
    bound = 7 * layers * bu.BF16 / 2
    off = lambda a, b: float((a.double().cpu() - b).norm() / b.norm())  # noqa: E731
    assert off(net.forward(x), y.detach()) <= bound
    assert off(net.backward(x, dy), leaf.grad) <= bound
    for i, layer in enumerate(w):
        for k, v in layer.items():
            assert off(net.grad[i][k], v.grad) <= bound, (i, k)


def test_updates():
    """Two of them: of the gradients, and of momenta that hold both."""
    net, x, dy = stack(70, 2)
    momentum = [{k: 0.0 for k in residual_stream.MATRICES} for _ in range(2)]
    for _ in range(2):
        net.forward(x)
        net.backward(x, dy)
        before = [{k: v.double().cpu().numpy() for k, v in layer.items()} for layer in net.master]
        grad = [{k: v.double().cpu().numpy() for k, v in layer.items()} for layer in net.grad]
        net.update(0.125, 0.5)
        for i in range(2):
            for k, v in net.master[i].items():
                got = v.double().cpu().numpy()
                assert not net.grad[i][k].any() and np.array_equal(net.w[i][k].double().cpu().numpy(), v.bfloat16().double().cpu().numpy())
                if v.dim() == 1:
                    assert np.abs(got - (before[i][k] - 0.125 * grad[i][k])).max() <= 4 * bu.FP32 * (np.abs(before[i][k]) + np.abs(grad[i][k])).max()
                    continue
                momentum[i][k] = 0.5 * momentum[i][k] + grad[i][k]
                want, bound = ru.ortho_bound(momentum[i][k], 5, None, 1e-7)
                # the momentum is rounded to fp32 and so is the weight's sum
                assert np.linalg.norm(got - (before[i][k] - 0.125 * want)) <= 0.125 * bound * 1.01 + 4 * bu.FP32 * np.linalg.norm(before[i][k])


def test_a_captured_step():
    """Forward, backward and update in one graph, replayed with the calls' own work between: the bits of the calls one by one."""
    (net, x, dy), (twin, _, _) = stack(130, 3), stack(130, 3)

    def step(of):
        of.forward(x)
        of.backward(x, dy)
        of.update(0.0625)

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step(net)
    torch.cuda.current_stream().wait_stream(side)
    step(twin)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step(net)
    for _ in range(3):
        graph.replay()
        torch.cuda.synchronize()
        step(twin)
        torch.cuda.synchronize()
        assert torch.equal(net.y, twin.y)
        for a, b in zip(net.master + net.momentum, twin.master + twin.momentum):
            assert all(torch.equal(a[k], b[k]) for k in a)
