"""The sizes of ortho_plans.py still take the ways that they stand for, and there is one for every way."""
import ortho_plans as kinds


def test_symmetric_products(tmp_path):
    plans = kinds.Plans(tmp_path)
    got = plans.of([size for size, *_ in kinds.SYMMETRIC])
    assert got == [tuple(names) for _, *names in kinds.SYMMETRIC]
    assert plans.names() == {names[0] for _, *names in kinds.SYMMETRIC}  # no way is left out
    assert {names[1] for _, *names in kinds.SYMMETRIC} <= plans.names()
    for (s, l), *_ in kinds.SYMMETRIC:
        assert all(sorted(-(-v // 64) * 64 for v in weight) == [s, l] for weight in kinds.weights_of(s, l))
