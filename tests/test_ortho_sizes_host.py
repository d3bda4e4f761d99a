"""The largest weights that the orthogonalised update takes, as axo_update.h has them."""
import pytest

import paper_2305_13525_amd as axo

WORKSPACE, BAD_SIZE = -7, -10


def P(K, N):
    return axo.Problem.make((1, 1, 1), (0, 0, 0), 64, K, N)


def at(n):
    return n << 40  # never dereferenced


# s x l, the larger sizes that are taken beside each s: s (l + 256) < 2^31 - 2^15, both multiples of 64
LARGEST = [(64, 33553600), (128, 16776640), (32768, 65216), (46208, 46208)]


@pytest.mark.parametrize("s,l", LARGEST)
def test_largest_weights_to_orthogonalise(s, l):
    call = lambda k, n: axo.axo_ortho(P(K=k, N=n), at(1), (n + 7) // 8 * 8, 0, 5, None, 0.0, at(2), (n + 7) // 8 * 8, at(3), 16, check=False)  # noqa: E731
    assert s * (l + 256) < 2 ** 31 - 2 ** 15 <= s * (l + 64 + 256)
    for k, n in ((s, l), (l, s), (s - 63, l - 63)):
        assert axo.axo_ortho_workspace_bytes(P(K=k, N=n)) > 0 and call(k, n) == WORKSPACE
    for k, n in ((s, l + 1), (l + 1, s), (s, l + 64)):
        assert axo.axo_ortho_workspace_bytes(P(K=k, N=n)) == 0 and call(k, n) == BAD_SIZE
