"""The orthogonalised update on the GPU against the 64-bit iteration: bit for bit where every rounding on the way is exact, within what rounding can do elsewhere."""
import ctypes

import numpy as np
import pytest

torch = pytest.importorskip("torch")
import block_util as bu
import residual_util as ru
import paper_2305_13525_amd as axo
from oracle import residual as orr

pytestmark = pytest.mark.gpu


def workspace(p):
    n = axo.axo_ortho_workspace_bytes(p)
    return torch.zeros(n, dtype=torch.uint8, device=bu.DEV), n


def ortho(g, steps=5, abc=None, wide=False, gap=0, eps=0.0, kept=None):
    k, n = g.shape
    p = bu.problem(0, k, n)
    G, O = bu.Mat(g, gap, wide), bu.Out(k, n, gap + 8)
    ws, size = kept or workspace(p)
    axo.axo_ortho(p, G.ptr, G.ld, int(wide), steps, abc, eps, O.ptr, O.ld, ws.data_ptr(), size, bu.stream())
    torch.cuda.synchronize()
    return O.result()


def rounded(a):
    return torch.from_numpy(a).float().bfloat16().double().numpy()  # the fp32 values here are exact


def half(a):
    return a.astype(np.float16).astype(np.float64)


def hadamard(n):
    h = np.ones((1, 1))
    while len(h) < n:
        h = np.block([[h, h], [h, -h]])
    return h


# rows x columns: below a tile, whole tiles, ragged ones, wide and tall, products of several workgroups to a tile (every other way of dealing tiles out: ortho_plans.py)
SHAPES = [(1, 1), (1, 9), (7, 3), (40, 40), (64, 64), (65, 64), (64, 130), (130, 70), (128, 512), (200, 200), (515, 259), (257, 1000), (64, 4096), (3000, 72), (1000, 1030),
          (640, 2500), (2049, 1500), (60, 5000), (6000, 100), (128, 17000), (250, 4500), (9000, 200)]


@pytest.mark.parametrize("k,n", SHAPES)
@pytest.mark.parametrize("wide", [False, True])
def test_places(k, n, wide):
    """One step of 2 + (X X^T) / 2 + (X X^T)^2 / 4 on +-1 in the rows and columns of a Hadamard matrix, some rows twice, strewn over a matrix of zeros.  Its norm is a power of two and
    its Gram matrix all of zeros and one power of two, so that the one thing that is rounded ahead of the result is Q, whose diagonal runs from 2 down to 4^-s: to fp16.  With that,
    every element has to be the one that is due."""
    rng = np.random.default_rng(k * 7 + n)
    a, b = int(np.log2(k)), int(np.log2(n))
    b -= (a + b) % 2
    if b < 0:
        a, b = a - 1, 0
    rows, cols = 2 ** a, 2 ** b
    h = hadamard(max(rows, cols))
    block = h[:rows, :cols] if rows >= cols else h[rng.integers(0, max(1, cols // 2), rows)][:, :cols]
    if rows >= cols and cols > 1:  # columns twice
        block = h[:rows][:, rng.integers(0, max(1, rows // 2), cols)]
    at = np.sort(rng.permutation(k)[:rows]), np.sort(rng.permutation(n)[:cols])
    g = np.zeros((k, n))
    g[np.ix_(*at)] = block * np.exp2(rng.integers(-20, 20))
    abc = [2.0, 0.5, 0.25]
    x = (g.T if k > n else g) / np.linalg.norm(g)
    m = x @ x.T
    q = half(2.0 * np.eye(len(x)) + 0.5 * m + 0.25 * m @ m)
    want = q @ x  # sums of numbers of 11 bits, within a factor of 2^13 of each other: fp32 holds them
    back = lambda y: rounded(y.T if k > n else y)  # noqa: E731
    got = ortho(g, 1, abc, wide, 8)
    assert np.array_equal(got, back(want))
    # with steps around it that change nothing but round X to fp16, in which it is held as a power of two times its values, through both buffers
    scale = 2.0 ** min(13, int(0.5 * np.log2(k * n)))
    assert np.array_equal(ortho(g, 4, [1.0, 0.0, 0.0] * 2 + abc + [1.0, 0.0, 0.0], wide), back(half(want * scale) / scale))


@pytest.mark.parametrize("k,n", [(3970, 4200), (4300, 3900)])
def test_places_of_many_tiles(k, n):
    """More tiles of 128 rows than a round of them takes: others go over the products then."""
    test_places(k, n, False)


@pytest.mark.parametrize("k,n", SHAPES)
@pytest.mark.parametrize("wide", [False, True])
def test_five_steps(k, n, wide):
    rng = np.random.default_rng(k + 3 * n)
    g = bu.draw(rng, k, n, 1e-3, 0.0, wide)
    got = ortho(g, 5, None, wide, 8 * (k % 2), eps=1e-7)
    want, bound = ru.ortho_bound(g, 5, None, 1e-7)
    assert np.isfinite(got).all()
    off = np.linalg.norm(got - want)
    assert off <= bound, (off, bound)
    # what a sum over all values hides: no row and no column is further off than all of it may be, spread evenly, five times over
    for axis in (0, 1):
        assert np.linalg.norm(got - want, axis=axis).max() <= 5 * bound / np.sqrt(min(k, n)) + 1e-12


def test_singular_values():
    """Five steps take singular values from 0.01 on to 0.6 to 1.3, and leave the vectors."""
    rng = np.random.default_rng(1)
    u, _, v = np.linalg.svd(rng.standard_normal((300, 200)), full_matrices=False)
    g = (u * np.geomspace(1.0, 0.05, 200)) @ v
    o = ortho(g, wide=True)
    s = np.linalg.svd(o, compute_uv=False)
    assert s.max() < 1.3 and s.min() > 0.6
    m = u.T @ o @ v.T
    assert np.abs(m - np.diag(np.diag(m))).max() < 0.02


@pytest.mark.parametrize("wide,exponent", [(True, -140), (True, 120), (False, -130), (False, 120)])
def test_any_magnitude(wide, exponent):
    """A power of two in G changes nothing, down to subnormal values and up to squares that fp32 does not hold: the same bits."""
    rng = np.random.default_rng(9)
    for k, n in [(40, 72), (300, 517)]:
        g = rng.integers(-3, 4, (k, n)).astype(np.float64)
        assert np.array_equal(ortho(g * 2.0 ** exponent, wide=wide), ortho(g, wide=wide))


def test_offsets_past_32_bits():
    """Rows of G and O a billion elements apart."""
    ld = (1 << 30) + 8
    for k, n in ((3, 1000), (3, 70)):
        g = bu.draw(np.random.default_rng(11), k, n)
        far = [torch.empty((k - 1) * ld + 1024, dtype=torch.bfloat16, device=bu.DEV) for _ in range(2)]
        rows = [t.as_strided((k, n), (ld, 1)) for t in far]
        rows[0].copy_(torch.from_numpy(g).bfloat16())
        p = bu.problem(0, k, n)
        ws, size = workspace(p)
        axo.axo_ortho(p, far[0].data_ptr(), ld, 0, 5, None, 0.0, far[1].data_ptr(), ld, ws.data_ptr(), size, bu.stream())
        assert np.array_equal(rows[1].double().cpu().numpy(), ortho(g))


def test_one_workspace_for_all_sizes():
    """Calls of several sizes, whose products are cut in different ways, one behind the other on one workspace."""
    rng = np.random.default_rng(10)
    sizes = [(1024, 4096), (515, 259), (1500, 6144), (64, 64), (200, 900), (100, 6000), (7000, 250)]
    kept = max((workspace(bu.problem(0, k, n)) for k, n in sizes), key=lambda w: w[1])
    g = [bu.draw(rng, k, n) for k, n in sizes]
    want = [ortho(v) for v in g]
    for _ in range(2):
        for v, w in zip(g, want):
            assert np.array_equal(ortho(v, kept=kept), w)


def test_coefficients_of_each_step():
    rng = np.random.default_rng(2)
    g = bu.draw(rng, 100, 180)
    abc = [6.0, -20.0, 20.0, 1.0, -0.9, 0.0, 1.875, -1.25, 0.375]
    got = ortho(g, 3, abc)
    want, bound = ru.ortho_bound(g, 3, abc)
    assert np.linalg.norm(got - want) <= bound
    assert np.linalg.norm(got - orr.ortho(g, 3, abc[3:6] + abc[:3] + abc[6:])) > 4 * bound  # another order is another result


@pytest.mark.parametrize("size", [1e-30, 1e-12, 1.0, 1e15, 1e30])
def test_any_size_of_gradient(size):
    """The squares of neither end are fp32 numbers."""
    rng = np.random.default_rng(3)
    g = bu.draw(rng, 70, 90, 1.0, 0.0, True)
    scale = 2.0 ** int(np.log2(size))
    assert np.array_equal(ortho(g * scale, wide=True), ortho(g, wide=True))


def test_zeros_and_eps():
    z = np.zeros((70, 90))
    assert not ortho(z).any() and not ortho(z, eps=1e-7).any()
    rng = np.random.default_rng(4)
    g = bu.draw(rng, 70, 90)
    got = ortho(g, 1, [1.0, 0.0, 0.0], eps=100.0)
    want = g / (np.linalg.norm(g) + 100.0)
    assert np.abs(got - want).max() <= (bu.BF16 + 2 * ru.FP16) * np.abs(want).max()


@pytest.mark.parametrize("bad", [np.inf, np.nan])
def test_infinities_and_nans(bad):
    """They show, and are gone with the next call on the workspace."""
    rng = np.random.default_rng(5)
    g = bu.draw(rng, 70, 200)
    kept = workspace(bu.problem(0, 70, 200))
    clean = ortho(g, kept=kept)
    h = g.copy()
    h[3, 5] = bad
    k, n = g.shape
    G, O = bu.Mat(h), bu.Out(k, n)
    axo.axo_ortho(bu.problem(0, k, n), G.ptr, G.ld, 0, 5, None, 0.0, O.ptr, O.ld, kept[0].data_ptr(), kept[1], bu.stream())
    assert np.isnan(O.result()).all()
    assert np.array_equal(ortho(g, kept=kept), clean)


def test_one_large_value():
    """A gradient that is all in one place: singular value 1, the largest that X can have, in one element."""
    for k, n in ((4096, 4096), (33, 65)):
        g = np.zeros((k, n))
        g[k // 2, n // 3] = -3.0
        got = ortho(g)
        v = 1.0
        for _ in range(5):
            v = orr.QUINTIC[0] * v + orr.QUINTIC[1] * v ** 3 + orr.QUINTIC[2] * v ** 5
        assert abs(got[k // 2, n // 3] + v) <= 0.01 and np.count_nonzero(got) == 1


@pytest.mark.parametrize("k,n", [(64, 4096), (515, 259), (640, 2500), (1000, 1030)])
def test_same_bits_on_any_stream_and_in_graphs(k, n):
    rng = np.random.default_rng(6)
    g = bu.draw(rng, k, n)
    first = ortho(g)
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        assert np.array_equal(first, ortho(g))
    p = bu.problem(0, k, n)
    G, O = bu.Mat(g), bu.Out(k, n)
    ws, size = workspace(p)
    call = lambda: axo.axo_ortho(p, G.ptr, G.ld, 0, 5, None, 1e-7, O.ptr, O.ld, ws.data_ptr(), size, bu.stream())  # noqa: E731
    call()
    torch.cuda.synchronize()
    graphs = [torch.cuda.CUDAGraph() for _ in range(2)]  # on one workspace
    for graph in graphs:
        with torch.cuda.graph(graph):
            call()
    for turn in range(3):
        G.view().copy_(torch.from_numpy(np.roll(g, turn, axis=0)).bfloat16())
        call()
        torch.cuda.synchronize()
        eager = O.view().clone()
        for graph in graphs:
            O.flat.fill_(float("nan"))
            graph.replay()
            torch.cuda.synchronize()
            assert torch.equal(eager, O.view()), turn


def test_coefficients_are_read_before_the_call_returns():
    rng = np.random.default_rng(7)
    g = bu.draw(rng, 256, 512)
    want = ortho(g, 2, [2.0, -1.5, 0.5] * 2)
    p = bu.problem(0, 256, 512)
    G, O = bu.Mat(g), bu.Out(256, 512)
    ws, size = workspace(p)
    abc = (ctypes.c_float * 6)(*[2.0, -1.5, 0.5] * 2)
    L = axo.update._lib()
    assert L.axo_ortho(ctypes.byref(p), G.ptr, G.ld, 0, 2, abc, 0.0, O.ptr, O.ld, ws.data_ptr(), size, bu.stream()) == 0
    abc[0] = abc[3] = float("nan")
    torch.cuda.synchronize()
    assert np.array_equal(O.result(), want)
