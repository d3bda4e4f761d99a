"""The product with a residual on 64 x 128 tiles and on 256-row ones, rows of X fetched by whole cache lines or not, outputs on cache lines or straddling them, against the 64-bit
definition.  More than 2048 tokens and no workspace: whole tiles, of the kinds of axo_fc_fwd but that 64 x 128 ones stand for 128 x 64 ones."""
import pytest

torch = pytest.importorskip("torch")
import block_util as bu
import test_fc_add_gpu as add
import paper_2305_13525_amd as axo

pytestmark = pytest.mark.gpu
WIDE, TALL, WHOLE = axo.AXO_KERNEL_TILES_64_128, axo.AXO_KERNEL_TILES_128_64, axo.AXO_KERNEL_TILES_256

# the kind, whether rows of X are fetched by whole lines -> tokens x in-features x out-features
SIZES = [(TALL, False, (2752, 1024, 448)), (TALL, False, (2745, 1024, 437)), (TALL, True, (2745, 1000, 437)), (TALL, True, (2748, 3569, 429)), (TALL, True, (2752, 1032, 448)), (WHOLE, True, (2304, 1608, 4352)),
         (WHOLE, False, (2304, 1600, 4352)), (WHOLE, True, (2300, 1603, 4333))]


@pytest.mark.parametrize("kind,by_lines,size", SIZES)
@pytest.mark.parametrize("wide", [False, True])
def test_forward(kind, by_lines, size, wide):
    m, k, n = size
    d = add.inputs(m, k, n, sum(size), wide)
    X, W, p = bu.Mat(d["x"]), bu.Mat(d["w"]), bu.problem(*size)
    tiles = axo.axo_fc_tiles(p, axo.AXO_OP_FWD, X.ptr, X.ld, W.ptr, W.ld, W.ld)[1]
    assert m > 2048 and axo.axo_fc_add_workspace_bytes(p) == 0 and tiles == (1 << kind | (1 << 16 + kind if by_lines else 0))
    if kind == TALL:
        assert -(-m // 64) * -(-n // 128) <= 256  # 64 x 128 tiles then
    add.check_forward(d, 1, wide)
    add.check_forward(d, 3, wide, save=True)
    if kind == TALL:
        add.check_forward(d, 2, wide, save=True, gap=8)
