"""The orthogonalised update on the GPU at the accuracy that is documented, all of it and each row and column."""
import numpy as np
import pytest

torch = pytest.importorskip("torch")
import block_util as bu
import ortho_rounded as rounded
import test_ortho_gpu as update
from oracle import residual as orr

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("k,n,spread,documented", rounded.CASES)
def test_five_steps(k, n, spread, documented):
    g = rounded.gradient(k, n, spread)
    rounded.check(update.ortho(g, wide=True, gap=8 * (n % 2)), orr.ortho(g, 5), documented)


@pytest.mark.parametrize("k,n", rounded.SIZES)
def test_five_steps_of_a_bf16_gradient(k, n):
    g = bu.draw(np.random.default_rng(k + 5 * n), k, n, 1e-3)
    rounded.check(update.ortho(g, eps=1e-7), orr.ortho(g, 5, eps=1e-7), rounded.RANDOM)


def test_one_workspace_for_all_sizes():
    """Calls of several sizes, whose products are cut in different ways, one behind the other on one workspace, each against the definition."""
    sizes = [(1024, 4096), (515, 259), (1500, 6144), (64, 64), (200, 900), (100, 6000), (7000, 250), (2300, 1100)]
    kept = max((update.workspace(bu.problem(0, k, n)) for k, n in sizes), key=lambda w: w[1])
    g = [bu.draw(np.random.default_rng(k + n), k, n) for k, n in sizes]
    want = [orr.ortho(v, 5) for v in g]
    for _ in range(2):
        for v, w in zip(g, want):
            rounded.check(update.ortho(v, kept=kept), w, rounded.RANDOM)
