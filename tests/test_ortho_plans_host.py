"""The sizes of ortho_plans.py still take the ways that they stand for, and there is one for every way."""
import ortho_plans as kinds
import paper_2305_13525_amd as axo


def test_symmetric_products(tmp_path):
    plans = kinds.Plans(tmp_path)
    got = plans.of([size for size, *_ in kinds.SYMMETRIC])
    assert got == [tuple(names) for _, *names in kinds.SYMMETRIC]
    assert plans.names() == {names[0] for _, *names in kinds.SYMMETRIC}  # no way is left out
    assert {names[1] for _, *names in kinds.SYMMETRIC} <= plans.names()
    for (s, l), *_ in kinds.SYMMETRIC:
        assert all(sorted(-(-v // 64) * 64 for v in weight) == [s, l] for weight in kinds.weights_of(s, l))


def test_products_on_oblong_tiles():
    """Of the kinds of axo_fc_fwd, but that 64 x 128 tiles stand for 128 x 64 ones."""
    found = set()
    for s, l in kinds.OBLONG:
        for m, n in ((s, l), (l, s)):
            found.add(axo.axo_fc_kernel(axo.Problem.make((1, 1, 1), (0, 0, 0), m, s, n), axo.AXO_OP_FWD, s, n, n)[1])
            assert -(-m // 64) * -(-n // 128) <= 256
    assert found == {axo.AXO_KERNEL_TILES_64_128, axo.AXO_KERNEL_TILES_128_64}
