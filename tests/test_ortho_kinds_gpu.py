"""The orthogonalised update on every way in which its symmetric products are dealt out, bit for bit: inputs whose every value on the way is exact."""
import pytest

torch = pytest.importorskip("torch")
import block_util as bu
import ortho_plans as kinds
import paper_2305_13525_amd as axo

pytestmark = pytest.mark.gpu
# every plan, products on every kind of tile, and steps of one launch and of two
WEIGHTS = [w for size in [size for size, *_ in kinds.SYMMETRIC] + kinds.OBLONG for w in kinds.weights_of(*size)] + [(51, 600), (600, 51), (115, 1000), (1000, 115), (50, 5000), (5000, 50), (120, 16000), (16000, 120)]


def parity(v):
    """Whether the number of bits that are set is odd."""
    for shift in (16, 8, 4, 2, 1):
        v = v ^ (v >> shift)
    return v & 1


def case(k, n):
    """G, the coefficients of a step, and what it makes of G, all exact.

    +-1 in 2^a rows and 2^b columns of an even a + b, strewn over a matrix of zeros: |G| is a power of two, 2^((a+b)/2).  Seen from the side with fewer rows than columns, the rows are
    drawn from the first half of a Hadamard matrix's, some of them twice and more: X X^T, times r = 2^a, is 1 where two rows are alike and 0 elsewhere.  With 1/2 + r A + (r A)^2 / 4, Q has
    1 + d / 4 for two of d rows that are alike, 1/2 more on its diagonal, and Q X is X's row times 1/2 + d (1 + d / 4).  Sums that miss a step, add one twice or take one of another
    tile give something else: 1 / r A is a whole number only with all of its terms."""
    tall, s, l = k > n, min(k, n), max(k, n)
    a, b = s.bit_length() - 1, l.bit_length() - 1
    b -= (a + b) % 2
    if b < a:
        a, b = a - 1, a - 1
    gen = torch.Generator()
    gen.manual_seed(k * 7 + n)
    which = torch.randint(0, 2 ** b // 2, (2 ** a,), generator=gen)
    rows, cols = (torch.randperm(v, generator=gen)[:2 ** e].sort().values.to(bu.DEV) for v, e in ((s, a), (l, b)))
    alike = torch.bincount(which, minlength=2 ** b)[which].double().to(bu.DEV)
    sign = 1 - 2 * parity(which.int().to(bu.DEV)[:, None] & torch.arange(2 ** b, dtype=torch.int32, device=bu.DEV)[None, :]).float()
    g = torch.zeros((s, l), device=bu.DEV)
    g[rows[:, None], cols[None, :]] = sign
    factor = torch.zeros(s, dtype=torch.float64, device=bu.DEV)
    factor[rows] = 0.5 + alike * (1 + alike / 4)
    # the exactness that all rests on: the factors, and so every product with the one value that X has, are bf16 numbers and Q's values fp16 ones
    assert torch.equal(factor, factor.bfloat16().double()) and alike.max() <= 64
    want = (g.double() * (factor * 2.0 ** -((a + b) / 2))[:, None]).bfloat16()
    r = 2.0 ** a
    return (g.T if tall else g), [0.5, r, r * r / 4], (want.T if tall else want)


def ortho(g, abc, wide, gap):
    k, n = g.shape
    p = bu.problem(0, k, n)
    ld = (n + 7) // 8 * 8 + gap
    G = torch.full((k, ld), float("nan"), dtype=torch.float32 if wide else torch.bfloat16, device=bu.DEV)
    G[:, :n] = g
    O = torch.full((k, ld + 8), float("nan"), dtype=torch.bfloat16, device=bu.DEV)
    size = axo.axo_ortho_workspace_bytes(p)
    ws = torch.zeros(size, dtype=torch.uint8, device=bu.DEV)
    for _ in range(2):  # the second call finds what the first one left in the workspace
        O.fill_(float("nan"))
        axo.axo_ortho(p, G.data_ptr(), ld, int(wide), len(abc) // 3, abc, 0.0, O.data_ptr(), ld + 8, ws.data_ptr(), size, bu.stream())
    assert torch.isnan(O[:, n:]).all()
    return O[:, :n]


@pytest.mark.parametrize("k,n", WEIGHTS)
def test_places(k, n):
    g, abc, want = case(k, n)
    assert torch.equal(ortho(g, abc, k % 2 == 0, 8 * (n % 2)), want)
    # behind a step that changes nothing, out of the other buffer, and ahead of one: X is held in fp16 there, as a power of two times values of 7 bits
    assert torch.equal(ortho(g, [1.0, 0.0, 0.0] + abc + [1.0, 0.0, 0.0], k % 2 == 1, 0), want)
