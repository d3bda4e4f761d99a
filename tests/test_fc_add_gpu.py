"""The product with a residual in its epilogue and the gradient behind it, on the GPU, against the 64-bit definition."""
import numpy as np
import pytest

torch = pytest.importorskip("torch")
import block_util as bu
import residual_util as ru
import paper_2305_13525_amd as axo
from oracle import residual as orr

pytestmark = pytest.mark.gpu
SCALE = 0.75

# tokens x in-features x out-features: one of each, single tokens, a few, odd and ragged, tiles of each size and their edges, split reductions
SIZES = [(1, 1, 1), (1, 8, 8), (1, 64, 64), (1, 100, 33), (1, 1000, 520), (1, 4096, 192), (1, 65, 2049), (2, 70, 70), (3, 7, 5), (5, 512, 136), (8, 1032, 72),
         (15, 300, 100), (16, 256, 256), (17, 129, 65), (24, 520, 1000), (32, 64, 40), (33, 640, 130), (64, 192, 200), (65, 72, 64), (96, 256, 384),
         (100, 1000, 24), (128, 128, 128), (130, 130, 130), (200, 333, 77), (256, 256, 256), (257, 192, 320), (300, 64, 513), (512, 96, 640), (640, 200, 264),
         (1001, 259, 515), (1024, 128, 1024), (128, 5000, 136)]
WHOLE = [(512, 192, 4608), (2100, 136, 4400), (4099, 128, 2060), (2048, 64, 2048), (4096, 72, 4096)]


def inputs(m, k, n, seed, wide):
    rng = np.random.default_rng(seed)
    return {"x": bu.draw(rng, m, k), "w": bu.draw(rng, k, n, 1.5 / np.sqrt(max(k, 1))), "r": bu.draw(rng, m, n, 2.0, 0.5, wide), "bias": bu.draw(rng, 1, n, 0.5)[0],
            "dy": bu.draw(rng, m, n, 1.0, 0.0, wide)}


def forward(d, epilogue, wide, save=False, gap=0, p=None, scale=SCALE, r=True, off=0):
    """`off`: elements that the matrices start behind a cache line."""
    (m, k), n = d["x"].shape, d["w"].shape[1]
    p = p or bu.problem(m, k, n)
    X, W, R = bu.Mat(d["x"], gap), bu.Mat(d["w"], gap), bu.Mat(d["r"], gap + 8, wide) if r else None
    Y, Z = bu.Out(m, n, gap, wide), bu.Out(m, n, gap + 16) if save else None
    bias = bu.vec(d["bias"]) if epilogue else None
    size = axo.axo_fc_add_workspace_bytes(p)
    ws = torch.zeros(max(size, 16), dtype=torch.uint8, device=bu.DEV)
    axo.axo_fc_add(p, X.ptr, X.ld, W.ptr, W.ld, bu.ptr(bias), epilogue, bu.ptr(R), R.ld if r else 0, int(wide), scale, bu.ptr(Z), Z.ld if save else 0, Y.ptr, Y.ld,
                   ws.data_ptr(), size, bu.stream())
    torch.cuda.synchronize()
    assert not ws[:min(size, 1024)].any()  # the counters are back at zero
    return Y.result(), Z.result() if save else None


def check_forward(d, epilogue, wide, save=False, gap=0, p=None, scale=SCALE, adds=True):
    Y, Z = forward(d, epilogue, wide, save, gap, p, scale, adds)
    r = d["r"] if adds else None
    y, z = orr.fc_add(d["x"], d["w"], r, scale, epilogue, d["bias"] if epilogue and adds else None)
    by, bz = ru.fc_add_bounds(d["x"], d["w"], r, z, y, scale, epilogue, wide)
    bu.within(Y, y, by, "y")
    if save:
        bu.within(Z, z, bz, "z")


@pytest.mark.parametrize("m,k,n", [(1, 6400, 8192), (5, 8208, 6424), (16, 16384, 3208), (3, 5000, 5000), (9, 3500, 8000)])
def test_few_tokens_and_much_weight(m, k, n):
    """Weights that are read from memory, beyond 100 MB by rows of 256 bytes."""
    check_forward(inputs(m, k, n, m + k, m % 2 == 1), 1 + m % 3, m % 2 == 1, gap=8)


@pytest.mark.parametrize("m,k,n", SIZES)
@pytest.mark.parametrize("wide", [False, True])
def test_forward(m, k, n, wide):
    d = inputs(m, k, n, m + 7 * k + 11 * n, wide)
    check_forward(d, 0, wide)
    check_forward(d, 1, wide, gap=8)
    check_forward(d, 2, wide, save=True)
    check_forward(d, 3, wide, save=True, gap=8)


@pytest.mark.parametrize("m,k,n", WHOLE)
@pytest.mark.parametrize("wide", [False, True])
def test_forward_of_many_tiles(m, k, n, wide):
    d = inputs(m, k, n, m + 7 * k + 11 * n, wide)
    check_forward(d, 1, wide)
    check_forward(d, 3, wide, save=True, gap=8)


@pytest.mark.parametrize("m,k,n", [(1001, 1032, 520), (200, 2056, 136), (2048, 1000, 1032), (520, 600, 4104), (4000, 520, 4104)])
def test_rows_that_straddle_cache_lines(m, k, n):
    d = inputs(m, k, n, m, False)
    for gap in (0, 8, 56):
        check_forward(d, 1, False, gap=gap)


def test_empty_reduction_and_no_elements():
    d = inputs(5, 8, 24, 1, False)
    d["x"], d["w"] = d["x"][:, :0], d["w"][:0]
    for epilogue in (0, 1, 2, 3):
        check_forward(d, epilogue, False, save=epilogue > 1)
    for m, n in ((0, 24), (5, 0)):
        assert axo.axo_fc_add(bu.problem(m, 8, n), None if m == 0 else bu.Mat(np.zeros((m, 8))).ptr, 8, None if n == 0 else bu.Mat(np.zeros((8, n))).ptr, 24, None, 0, None, 0,
                              0, 1.0, None, 0, None, 0, None, 0, bu.stream()) == 0


def test_scales():
    d = inputs(33, 100, 72, 2, True)
    check_forward(d, 2, True, scale=-2.5)
    assert np.array_equal(forward(d, 2, True, scale=0.0)[0], d["r"])


@pytest.mark.parametrize("epilogue", [0, 1])
def test_split_reduction(epilogue):
    """On a grid that splits K the residual and the bias are added on the axis's first shard, which alone reads them."""
    d = inputs(64, 128, 72, 3, True)
    check_forward(d, epilogue, True, p=bu.problem(64, 256, 72, (2, 1, 1), (0, 0, 0)))
    check_forward(d, epilogue, True, p=bu.problem(64, 256, 72, (2, 1, 1), (1, 0, 0)), adds=False)
    check_forward(d, epilogue, True, p=bu.problem(64, 256, 72, (1, 2, 1), (0, 1, 0), 1), adds=False)


def test_infinities_and_nans_stay_where_they_are():
    """Of X in its row, of W in its column, of R in its place; what lies behind the matrices (NaN) nowhere."""
    for m, k, n in ((1, 300, 100), (70, 333, 130), (300, 100, 520)):
        d = inputs(m, k, n, 4, False)
        clean, _ = forward(d, 1, False)
        bad = {**d, "r": d["r"].copy(), "w": d["w"].copy()}
        bad["r"][0, 3], bad["w"][k // 2, 7] = np.inf, np.nan
        got, _ = forward(bad, 1, False)
        assert np.isinf(got[0, 3]) and np.isnan(got[:, 7]).all()
        rest = np.ones((m, n), bool)
        rest[0, 3] = rest[:, 7] = False
        assert np.array_equal(got[rest], clean[rest])


def test_operands_past_4_gib():
    """Rows of X and W half a gigabyte apart."""
    m, k, n, ld = 9, 20, 40, (1 << 28) + 8
    d = inputs(m, k, n, 5, False)
    big = torch.empty(19 * ld + 64, dtype=torch.bfloat16, device=bu.DEV)
    big.as_strided((k, n), (ld, 1)).copy_(torch.from_numpy(d["w"]).bfloat16())
    X, R, Y, p = bu.Mat(d["x"]), bu.Mat(d["r"]), bu.Out(m, n), bu.problem(m, k, n)
    size = axo.axo_fc_add_workspace_bytes(p)
    ws = torch.zeros(max(size, 16), dtype=torch.uint8, device=bu.DEV)
    bias = bu.vec(d["bias"])
    axo.axo_fc_add(p, X.ptr, X.ld, big.data_ptr(), ld, bias.data_ptr(), 1, R.ptr, R.ld, 0, SCALE, None, 0, Y.ptr, Y.ld, ws.data_ptr(), size, bu.stream())
    y, z = orr.fc_add(d["x"], d["w"], d["r"], SCALE, 1, d["bias"])
    bu.within(Y.result(), y, ru.fc_add_bounds(d["x"], d["w"], d["r"], z, y, SCALE, 1, False)[0])


@pytest.mark.parametrize("m,k,n", [(3, 72, 40), (3, 4096, 72)])
def test_stream_past_4_gib(m, k, n):
    """Rows of R, Y, Z and of the gradients a billion elements apart."""
    d, ld = inputs(m, k, n, 12, False), (1 << 30) + 8
    far = [torch.empty((m - 1) * ld + 1024, dtype=torch.bfloat16, device=bu.DEV) for _ in range(4)]
    R, Y, Z, dZ = (t.as_strided((m, n), (ld, 1)) for t in far)
    R.copy_(torch.from_numpy(d["r"]).bfloat16())
    X, W, p, bias = bu.Mat(d["x"]), bu.Mat(d["w"]), bu.problem(m, k, n), bu.vec(d["bias"])
    size = axo.axo_fc_add_workspace_bytes(p)
    ws = torch.zeros(max(size, 16), dtype=torch.uint8, device=bu.DEV)
    axo.axo_fc_add(p, X.ptr, X.ld, W.ptr, W.ld, bias.data_ptr(), 2, far[0].data_ptr(), ld, 0, SCALE, far[2].data_ptr(), ld, far[1].data_ptr(), ld, ws.data_ptr(), size, bu.stream())
    y, z = forward(d, 2, False, save=True)
    back = lambda t: t.double().cpu().numpy()  # noqa: E731
    assert np.array_equal(back(Y), y) and np.array_equal(back(Z), z)
    axo.axo_fc_add_dact(p, far[0].data_ptr(), ld, 0, far[2].data_ptr(), ld, 2, SCALE, far[3].data_ptr(), ld, bu.stream())
    want = SCALE * d["r"] * orr.act(z, 2)[1]
    bu.within(back(dZ), want, ru.dact_bound(d["r"], z, SCALE, 2, want))


@pytest.mark.parametrize("m,n", [(1, 1), (1, 8), (3, 7), (70, 333), (257, 1024), (1000, 520)])
@pytest.mark.parametrize("wide", [False, True])
def test_gradient(m, n, wide):
    d = inputs(m, 8, n, 6, wide)
    z = bu.draw(np.random.default_rng(7), m, n, 3.0)
    for epilogue in range(4):
        for gap in (0, 8):
            dY, Z, dZ = bu.Mat(d["dy"], gap, wide), bu.Mat(z, gap + 8), bu.Out(m, n, gap)
            has = epilogue >= 2
            axo.axo_fc_add_dact(bu.problem(m, 8, n), dY.ptr, dY.ld, int(wide), Z.ptr if has else None, Z.ld if has else 0, epilogue, SCALE, dZ.ptr, dZ.ld, bu.stream())
            want = SCALE * d["dy"] * orr.act(z, epilogue)[1]
            bu.within(dZ.result(), want, ru.dact_bound(d["dy"], z, SCALE, epilogue, want), epilogue)


def test_gradients_of_the_layer_against_differences():
    """dZ through the layer's products: the gradient of sum(y dy) along a direction of X, W, bias and R."""
    m, k, n = 40, 72, 56
    d = inputs(m, k, n, 8, True)
    rng = np.random.default_rng(9)
    v = {name: rng.standard_normal(d[name].shape) for name in ("x", "w", "bias", "r")}
    for epilogue in (1, 2, 3):
        p = bu.problem(m, k, n)
        _, z = forward(d, max(epilogue, 2), True, save=True)
        X, W, Z, dY, dZ, dX, dW = bu.Mat(d["x"]), bu.Mat(d["w"]), bu.Mat(z), bu.Mat(d["dy"], 0, True), bu.Out(m, n), bu.Out(m, k), bu.Out(k, n)
        has = epilogue >= 2
        axo.axo_fc_add_dact(p, dY.ptr, dY.ld, 1, Z.ptr if has else None, Z.ld if has else 0, epilogue, SCALE, dZ.ptr, dZ.ld, bu.stream())
        axo.axo_fc_dgrad(p, dZ.ptr, dZ.ld, W.ptr, W.ld, dX.ptr, dX.ld, None, 0, bu.stream())
        axo.axo_fc_wgrad(p, X.ptr, X.ld, dZ.ptr, dZ.ld, dW.ptr, dW.ld, None, 0, bu.stream())
        db = torch.zeros(n, device=bu.DEV)
        axo.axo_bias_grad(p, dZ.ptr, dZ.ld, db.data_ptr(), 0, bu.stream())
        torch.cuda.synchronize()
        parts = [dX.result() * v["x"], dW.result() * v["w"], db.double().cpu().numpy() * v["bias"], d["dy"] * v["r"]]
        loss = lambda t: (orr.fc_add(d["x"] + t * v["x"], d["w"] + t * v["w"], d["r"] + t * v["r"], SCALE, epilogue, d["bias"] + t * v["bias"])[0] * d["dy"]).sum()  # noqa: E731, B023
        slope = (loss(1e-5) - loss(-1e-5)) / 2e-5
        # Z, dZ and dX or dW are rounded to bf16 on the way, Z where the slope changes by at most 1.2 per unit
        dz = np.abs(SCALE * d["dy"])
        err_dz = dz * (bu.SLOPE * bu.BF16 + (1.2 * bu.BF16 * np.abs(z) if has else 0))
        bound = (err_dz @ np.abs(d["w"]).T * np.abs(v["x"])).sum() + (np.abs(d["x"]).T @ err_dz * np.abs(v["w"])).sum() + (err_dz.sum(axis=0) * np.abs(v["bias"])).sum()
        bound += bu.BF16 * (np.abs(parts[0]).sum() + np.abs(parts[1]).sum()) + 1e-5 * sum(np.abs(q).sum() for q in parts)
        assert abs(sum(q.sum() for q in parts) - slope) <= bound


@pytest.mark.parametrize("m,k,n", [(1, 8192, 256), (17, 2048, 192), (128, 5000, 136), (300, 256, 513), (1024, 512, 1032)])
def test_same_bits_on_any_stream_and_in_graphs(m, k, n):
    d = inputs(m, k, n, 10, False)
    first = forward(d, 3, False, save=True)
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        again = forward(d, 3, False, save=True)
    assert all(np.array_equal(a, b) for a, b in zip(first, again))
    p = bu.problem(m, k, n)
    X, W, R, dY = bu.Mat(d["x"]), bu.Mat(d["w"]), bu.Mat(d["r"]), bu.Mat(d["dy"])
    Y, Z, dZ = (bu.Out(m, n) for _ in range(3))
    bias = bu.vec(d["bias"])
    size = axo.axo_fc_add_workspace_bytes(p)
    ws = torch.zeros(max(size, 16), dtype=torch.uint8, device=bu.DEV)

    def both():
        axo.axo_fc_add(p, X.ptr, X.ld, W.ptr, W.ld, bias.data_ptr(), 3, R.ptr, R.ld, 0, SCALE, Z.ptr, Z.ld, Y.ptr, Y.ld, ws.data_ptr(), size, bu.stream())
        axo.axo_fc_add_dact(p, dY.ptr, dY.ld, 0, Z.ptr, Z.ld, 3, SCALE, dZ.ptr, dZ.ld, bu.stream())

    both()
    torch.cuda.synchronize()
    graphs = [torch.cuda.CUDAGraph() for _ in range(2)]  # on one workspace
    for g in graphs:
        with torch.cuda.graph(g):
            both()
    results = [Y.view(), Z.view(), dZ.view()]
    for turn in range(3):
        X.view().copy_(torch.from_numpy(np.roll(d["x"], turn, axis=1)).bfloat16())
        both()
        torch.cuda.synchronize()
        eager = [t.clone() for t in results]
        for g in graphs:
            for t in results:
                t.fill_(float("nan"))
            g.replay()
            torch.cuda.synchronize()
            assert all(torch.equal(a, b) for a, b in zip(eager, results)), turn
