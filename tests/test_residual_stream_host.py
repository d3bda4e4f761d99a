"""What examples/residual_stream.py refuses ahead of its first call: the library is given addresses, and cannot see that a buffer is too small."""
import os
import sys

import pytest

torch = pytest.importorskip("torch")
sys.path.insert(0, os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples"))
import residual_stream  # noqa: E402


class Called(Exception):
    pass


@pytest.fixture
def net(monkeypatch):
    """A stack in host memory, whose requests for a stream raise."""
    def called(*a, **k):
        raise Called

    monkeypatch.setattr(residual_stream, "DEV", "cpu")
    monkeypatch.setattr(torch.cuda, "current_stream", called)
    return residual_stream.Stream(8, 16, 24, 2)


def rows(n, width=16, dtype=torch.float32):
    return torch.zeros((n, width), dtype=dtype)


@pytest.mark.parametrize("x", [rows(9), rows(7), rows(8, 24), rows(8, dtype=torch.bfloat16), rows(8)[0], rows(8, 32)[:, ::2], rows(8, 18)[:, :16], rows(9)[:, :16].flatten()[1:129].view(8, 16)])
def test_refuses(net, x):
    with pytest.raises(ValueError):
        net.forward(x)
    net._forwarded = True
    with pytest.raises(ValueError):
        net.backward(x, rows(8))
    with pytest.raises(ValueError):
        net.backward(rows(8), x)


def test_takes_what_it_can_read(net):
    with pytest.raises(Called):
        net.forward(rows(8))
    with pytest.raises(ValueError):
        net.backward(rows(8), rows(8))  # ahead of a forward pass
    net._forwarded = True
    with pytest.raises(Called):
        net.backward(rows(8, 24)[:, :16], rows(8, 32)[:, 16:])


@pytest.mark.parametrize("sizes", [(8, 20, 24, 2), (8, 16, 20, 2), (8, 16, 24, 0)])
def test_refuses_sizes(net, sizes):
    with pytest.raises(ValueError):
        residual_stream.Stream(*sizes)
