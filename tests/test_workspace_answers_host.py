"""What the workspace query of the norms around a residual addition says of problems that its call refuses."""
import pytest

import paper_2305_13525_amd as axo

BAD_GRID, WORKSPACE = -1, -7


def P(T=64, K=32, N=48, grid=(1, 1, 1), coord=(0, 0, 0), transposed=0):
    return axo.Problem.make(grid, coord, T, K, N, transposed)


def at(n):
    return n << 40  # never dereferenced


def resnorm_bwd(p, ws, ws_bytes):
    return axo.axo_resnorm_bwd(p, at(1), 32, None, 0, at(2), 32, at(3), 32, 0, 1, None, None, None, 1.0, 1, None, at(4), at(5), 32, at(6), 32, at(7), None, None, None, None, 0, ws,
                               ws_bytes, check=False)


@pytest.mark.parametrize("grid,transposed", [((2, 1, 1), 0), ((1, 2, 1), 1), ((4, 2, 2), 0)])
def test_split_widths_have_no_workspace_of_the_norms(grid, transposed):
    p = P(grid=grid, transposed=transposed)
    assert resnorm_bwd(p, at(8), 1 << 40) == BAD_GRID
    assert axo.axo_resnorm_workspace_bytes(p) == 0


@pytest.mark.parametrize("grid,transposed", [((1, 2, 1), 0), ((2, 1, 1), 1), ((1, 1, 4), 0)])
def test_whole_widths_have_one(grid, transposed):
    p = P(grid=grid, transposed=transposed)
    n = axo.axo_resnorm_workspace_bytes(p)
    assert n > 0 and resnorm_bwd(p, at(8), n - 1) == WORKSPACE
