"""What is documented of the orthogonalised update's accuracy holds for the roundings that it has, and would not with X, A and Q in bf16."""
import numpy as np
import pytest

import ortho_rounded as rounded
from oracle import residual as orr


SMALL = [c for c in rounded.CASES if c[0] * c[1] <= 300000]  # quick on the host


@pytest.mark.parametrize("k,n,spread,documented", SMALL)
def test_roundings(k, n, spread, documented):
    g = rounded.gradient(k, n, spread)
    want = orr.ortho(g, 5)
    rounded.check(rounded.to(rounded.BF, rounded.update(g, rounded.HALF)), want, documented)
    with pytest.raises(AssertionError):
        rounded.check(rounded.to(rounded.BF, rounded.update(g, rounded.BF)), want, documented)


@pytest.mark.parametrize("spread,least,most", [(10.0, 0.0005, 0.0015), (30.0, 0.001, 0.002), (100.0, 0.0015, 0.0045), (1000.0, 0.003, 0.012)])
def test_documented_figures(spread, least, most):
    for k, n in ((64, 4096), (128, 512), (300, 310)):
        g = rounded.gradient(k, n, spread)
        want = orr.ortho(g, 5)
        assert least <= np.linalg.norm(rounded.update(g, rounded.HALF) - want) / np.linalg.norm(want) <= most


def test_a_row_that_is_lost_shows():
    for k, n, spread, documented in SMALL[::4]:
        want = orr.ortho(rounded.gradient(k, n, spread), 5)
        for axis, length in enumerate(want.shape):
            got = want.copy()
            got[(slice(None),) * axis + (length // 2,)] = 0.0
            with pytest.raises(AssertionError):
                rounded.check(got, want, documented)
