"""The product with a residual where workgroups share a tile's reduction: tiles whose waves split it, and 128 x 128 tiles in slices that a second launch adds up and finishes,
against the 64-bit definition."""
import numpy as np
import pytest

torch = pytest.importorskip("torch")
import add_slices as kinds
import block_util as bu
import test_fc_add_gpu as add
import paper_2305_13525_amd as axo

pytestmark = pytest.mark.gpu
SLICES = [size for tiles, size in kinds.SLICED if tiles == kinds.WHOLE]


@pytest.mark.parametrize("tiles,size", kinds.SLICED)
@pytest.mark.parametrize("wide", [False, True])
def test_forward(tiles, size, wide):
    assert {f[:2] for f in kinds.sliced_on(*size)} == {tiles}
    d = add.inputs(*size, sum(size), wide)
    add.check_forward(d, 0, wide)
    add.check_forward(d, 1, wide, gap=8)
    add.check_forward(d, 2, wide, save=True, gap=64)
    add.check_forward(d, 3, wide, save=True, gap=8)


@pytest.mark.parametrize("size", [(287, 9235, 745), (300, 8192, 512)])
def test_shards_of_a_split_reduction(size):
    """The residual and the bias are added, in the second launch, by the shard whose coordinate is 0."""
    m, k, n = size
    d = add.inputs(m, k, n, 3, True)
    for ix in (0, 1):
        p = bu.problem(m, 2 * k, n, (2, 1, 1), (ix, 0, 0))
        assert axo.axo_fc_add_workspace_bytes(p) == axo.axo_fc_add_workspace_bytes(bu.problem(m, k, n))
        add.check_forward(d, 1, True, p=p, adds=ix == 0)


@pytest.mark.parametrize("size", [(707, 6246, 270), (300, 8192, 512)])
def test_infinities_and_nans_stay_where_they_are(size):
    m, k, n = size
    d = add.inputs(m, k, n, 4, False)
    clean, _ = add.forward(d, 1, False)
    bad = {**d, "r": d["r"].copy(), "w": d["w"].copy(), "x": d["x"].copy()}
    bad["r"][0, 3], bad["w"][k // 2, 7], bad["x"][m - 1, k - 1] = np.inf, np.nan, np.nan
    got, _ = add.forward(bad, 1, False)
    assert np.isinf(got[0, 3]) and np.isnan(got[:, 7]).all() and np.isnan(got[m - 1]).all()
    rest = np.ones((m, n), bool)
    rest[0, 3] = rest[:, 7] = rest[m - 1] = False
    assert np.array_equal(got[rest], clean[rest])


def test_one_workspace_for_all_sizes():
    """Calls whose tiles are shared in different ways, one behind the other on one workspace."""
    sizes = [(33, 8192, 200), (300, 8192, 512), (1, 9416, 933), (707, 6246, 270), (1, 13373, 3797), (287, 9235, 745), (1, 6130, 1020)]
    problems = [bu.problem(*s) for s in sizes]
    need = max(axo.axo_fc_add_workspace_bytes(p) for p in problems)
    ws = torch.zeros(need, dtype=torch.uint8, device=bu.DEV)
    made = [add.inputs(*s, sum(s), False) for s in sizes]
    want = [add.forward(d, 1, False)[0] for d in made]
    for _ in range(2):
        for (m, k, n), p, d, w in zip(sizes, problems, made, want):
            X, W, R, Y, bias = bu.Mat(d["x"]), bu.Mat(d["w"]), bu.Mat(d["r"]), bu.Out(m, n), bu.vec(d["bias"])
            axo.axo_fc_add(p, X.ptr, X.ld, W.ptr, W.ld, bias.data_ptr(), 1, R.ptr, R.ld, 0, add.SCALE, None, 0, Y.ptr, Y.ld, ws.data_ptr(), need, bu.stream())
            assert np.array_equal(Y.result(), w)


@pytest.mark.parametrize("size", [(287, 9235, 745), (640, 4096, 256)])
def test_same_bits_on_any_stream_and_in_graphs(size):
    add.test_same_bits_on_any_stream_and_in_graphs(*size)
