"""The sizes of add_slices.py still take the ways that they stand for, and there is one for every way."""
import pytest

import add_slices as kinds


@pytest.mark.parametrize("tiles,size", kinds.SLICED)
def test_products_that_share_a_tile(tiles, size):
    found = kinds.sliced_on(*size)
    assert len(found) == 1 and {f[:2] for f in found} == {tiles}, found


def test_every_kind_of_tile_is_shared():
    assert {t for t, _ in kinds.SLICED} == set(kinds.FEW) | {kinds.WHOLE}
    assert {min(s) for s in (kinds.sliced_on(*size) for t, size in kinds.SLICED if t == kinds.WHOLE)} >= {(*kinds.WHOLE, 2), (*kinds.WHOLE, 16)}
