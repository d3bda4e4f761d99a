"""What examples/gated_mlp.py refuses ahead of its first call: the library is given addresses, and cannot see that a buffer is too small."""
import os
import sys

import pytest

torch = pytest.importorskip("torch")
sys.path.insert(0, os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples"))
import gated_mlp  # noqa: E402


class Called(Exception):
    pass


@pytest.fixture
def net(monkeypatch):
    """A sublayer in host memory, whose calls of the library and requests for a stream raise."""
    def called(*a, **k):
        raise Called

    monkeypatch.setattr(gated_mlp, "DEV", "cpu")
    monkeypatch.setattr(torch.cuda, "current_stream", called)
    return gated_mlp.GatedMLP(8, 16, 24)


def rows(n, width=16, dtype=torch.bfloat16):
    return torch.zeros((n, width), dtype=dtype)


@pytest.mark.parametrize("x", [rows(9), rows(8, 24), rows(8, dtype=torch.float32), rows(8)[0], rows(8, 32)[:, ::2], rows(16, 8).t()[:, :16]])
def test_forward_refuses(net, x):
    with pytest.raises(ValueError):
        net.forward(x)
    net._forwarded = 8
    with pytest.raises(ValueError):
        net.backward(x, rows(8))
    with pytest.raises(ValueError):
        net.backward(rows(8), x)


def test_forward_takes_as_many_tokens_as_there_are_buffers_for(net):
    for n in (0, 1, 8):
        with pytest.raises(Called):
            net.forward(rows(n))


def test_backward_belongs_to_the_last_forward_pass(net):
    for forwarded, x, dy in ((0, 8, 8), (4, 8, 8), (8, 8, 4), (8, 4, 4)):
        net._forwarded = forwarded
        with pytest.raises(ValueError):
            net.backward(rows(x), rows(dy))
    with pytest.raises(Called):
        net._forwarded = 8
        net.backward(rows(8), rows(8))
