"""The gated feed-forward block on the GPU, forward and backward, against the 64-bit definition."""
import numpy as np
import pytest

torch = pytest.importorskip("torch")
import block_util as bu
import paper_2305_13525_amd as axo
from oracle import block as ob

pytestmark = pytest.mark.gpu

# tokens x width x inner width: one of each, single tokens, a few, odd and ragged, tiles of each size and their edges
SIZES = [(1, 1, 1), (1, 8, 8), (1, 64, 64), (1, 100, 33), (1, 1000, 520), (1, 4096, 192), (1, 65, 2049), (2, 70, 70), (3, 7, 5), (5, 512, 136), (8, 1032, 72),
         (15, 300, 100), (16, 256, 256), (17, 129, 65), (24, 520, 1000), (32, 64, 40), (33, 640, 130), (64, 192, 200), (65, 72, 64), (96, 256, 384),
         (100, 1000, 24), (128, 128, 128), (130, 130, 130), (200, 333, 77), (256, 256, 256), (257, 192, 320), (300, 64, 513), (512, 96, 640), (640, 200, 264),
         (1001, 259, 515), (1024, 128, 1024)]
WHOLE = [(512, 192, 2304), (2100, 136, 2200), (4099, 128, 1030)]


def inputs(m, k, f, seed):
    rng = np.random.default_rng(seed)
    sw = 1.5 / np.sqrt(max(k, 1))  # G and U of deviation 1.5
    return {"x": bu.draw(rng, m, k), "wg": bu.draw(rng, k, f, sw), "wu": bu.draw(rng, k, f, sw), "bg": bu.draw(rng, 1, f, 0.5)[0],
            "bu": bu.draw(rng, 1, f, 0.5)[0]}


def workspace(p):
    n = axo.axo_gated_workspace_bytes(p)
    return torch.zeros(max(n, 16), dtype=torch.uint8, device=bu.DEV), n


def forward(d, kind, save=True, bias=(True, True), gap=0, p=None):
    (m, k), f = d["x"].shape, d["wg"].shape[1]
    p = p or bu.problem(m, k, f)
    X, Wg, Wu = bu.Mat(d["x"], gap), bu.Mat(d["wg"], gap), bu.Mat(d["wu"], gap)
    H = bu.Out(m, f, gap)
    G, U = (bu.Out(m, f, gap + 8), bu.Out(m, f, gap + 8)) if save else (None, None)
    bg, bv = bu.vec(d["bg"]) if bias[0] else None, bu.vec(d["bu"]) if bias[1] else None
    ws, n = workspace(p)
    axo.axo_gated_fwd(p, X.ptr, X.ld, Wg.ptr, Wu.ptr, Wg.ld, bu.ptr(bg), bu.ptr(bv), kind, bu.ptr(G), bu.ptr(U), G.ld if save else 0, H.ptr, H.ld,
                      ws.data_ptr(), n, bu.stream())
    torch.cuda.synchronize()
    assert not ws[:min(n, 1024)].any()  # the counters are back at zero
    return H.result(), G.result() if save else None, U.result() if save else None


def check_forward(d, kind, save=True, bias=(True, True), gap=0, p=None, with_bias=None):
    got = forward(d, kind, save, bias, gap, p)
    bg, bv = (d[n] if (b if with_bias is None else with_bias) else None for n, b in zip(("bg", "bu"), bias))
    h, g, u = ob.gated_fwd(d["x"], d["wg"], d["wu"], kind, bg, bv)
    bounds = bu.gated_fwd_bounds(d["x"], d["wg"], d["wu"], g, u, ob.gate(g, kind)[0])
    for a, want, bound, name in zip(got, (h, g, u), bounds, "HGU"):
        if a is not None:
            bu.within(a, want, bound, name)
    return got


@pytest.mark.parametrize("m,k,f", SIZES)
def test_forward(m, k, f):
    d = inputs(m, k, f, m + 7 * k + 11 * f)
    kind = (m + k + f) % 3
    a = check_forward(d, kind, True, (True, True), 0)
    b = check_forward(d, kind, False, (True, True), 0)
    assert np.array_equal(a[0], b[0])  # H does not depend on what else is stored
    check_forward(d, (kind + 1) % 3, True, (False, True), 8)
    check_forward(d, (kind + 2) % 3, False, (True, False), 56)


@pytest.mark.parametrize("m,k,f", WHOLE)
@pytest.mark.parametrize("kind", [0, 1, 2])
def test_forward_whole_tiles(m, k, f, kind):
    check_forward(inputs(m, k, f, kind), kind, kind != 1, (kind != 2, kind != 2))


# (op, rows, columns, whether workgroups share a tile) -> tokens x width x inner width that run on such tiles, whole chunks and odd ones
VARIANTS = [
    (0, 16, 32, False, (1, 704, 8)), (0, 16, 32, False, (1, 663, 9)), (0, 16, 32, True, (1, 2048, 8)), (0, 16, 32, True, (2, 2016, 9)),
    (0, 16, 64, False, (1, 64, 8232)), (0, 16, 64, False, (1, 8, 8486)), (0, 16, 64, True, (2, 5120, 1336)), (0, 16, 64, True, (1, 4095, 1566)),
    (0, 16, 128, False, (1, 3328, 16608)), (0, 16, 128, True, (1, 4618, 10914)),
    (0, 32, 32, False, (290, 1280, 8)), (0, 32, 32, False, (268, 975, 10)), (0, 32, 32, True, (321, 2304, 8)), (0, 32, 32, True, (270, 2004, 10)),
    (0, 64, 32, False, (1, 64, 8)), (0, 64, 32, False, (1, 8, 9)), (0, 64, 64, False, (3, 1024, 14565)), (0, 64, 64, False, (1, 964, 14028)),
    (0, 64, 64, False, (130, 256, 4200)), (0, 64, 64, False, (140, 250, 4203)), (1, 64, 128, False, (130, 640, 8300)), (1, 64, 128, False, (135, 643, 8303)),
    (0, 128, 64, False, (17, 64, 8880)), (0, 128, 64, False, (20, 8, 8199)), (0, 256, 128, False, (133, 64, 9416)), (0, 256, 128, False, (137, 8, 9259)),
    (1, 16, 32, False, (2, 1920, 8)), (1, 16, 32, False, (1, 1840, 9)), (1, 16, 32, True, (1, 2048, 8)), (1, 16, 32, True, (2, 2016, 9)),
    (1, 32, 32, False, (1, 768, 8)), (1, 32, 32, False, (1, 705, 9)), (1, 32, 32, True, (351, 2112, 8)), (1, 32, 32, True, (258, 2073, 9)),
    (1, 64, 64, False, (1, 64, 8)), (1, 64, 64, False, (1, 8, 9)), (1, 64, 128, False, (23, 1088, 19000)), (1, 64, 128, False, (20, 961, 18788)),
    (1, 128, 128, False, (330, 64, 6000)), (1, 128, 128, False, (325, 8, 6007)), (1, 256, 256, False, (700, 64, 13824)), (1, 256, 256, False, (697, 8, 13801)),
    (1, 64, 64, False, (21, 64, 17144)), (1, 64, 64, False, (19, 8, 16533)), (1, 64, 64, False, (144, 64, 16512)), (1, 64, 64, False, (129, 8, 17245)),
    (2, 16, 32, False, (2, 64, 840)), (2, 16, 32, False, (1, 9, 806)), (2, 16, 32, True, (1, 64, 968)), (2, 16, 32, True, (1, 9, 961)),
    (2, 32, 32, False, (1, 64, 360)), (2, 32, 32, False, (2, 9, 354)), (2, 32, 32, True, (294, 64, 992)), (2, 32, 32, True, (272, 10, 962)),
    (2, 64, 64, False, (1, 64, 8)), (2, 64, 64, False, (1, 9, 8)), (2, 64, 128, False, (3904, 320, 504)), (2, 64, 128, False, (3678, 282, 481)),
    (2, 128, 128, False, (85, 8640, 8)), (2, 128, 128, False, (82, 8423, 8)), (2, 256, 256, False, (404, 8384, 8)), (2, 256, 256, False, (397, 8315, 8)),
    (0, 128, 64, True, (408, 2880, 8)), (0, 128, 64, True, (409, 2922, 9)), (0, 128, 64, True, (300, 6400, 328)), (0, 128, 64, True, (310, 6411, 333)),
    (1, 128, 128, True, (1390, 6720, 72)), (1, 128, 128, True, (1407, 6628, 68)), (2, 128, 128, True, (112, 704, 4720)), (2, 128, 128, True, (1065, 99, 2956)),
    (3, 128, 128, True, (4701, 64, 120)), (3, 128, 128, True, (4534, 114, 131)), (3, 128, 128, True, (5784, 640, 752))]


@pytest.mark.parametrize("op,rows,cols,shared,size", VARIANTS)
def test_every_kind_of_tiles(op, rows, cols, shared, size):
    m, k, f = size
    p = bu.problem(m, f, k) if op == axo.AXO_GATED_OP_DGRAD_ACT else bu.problem(m, k, f)
    got = axo.axo_gated_tiles(p, op)[1]
    assert got[:2] == (rows, cols) and (got[2] > 1) == shared, got
    kind, gap = (m + f) % 3, (0, 8)[(k + f) % 2]
    if op == axo.AXO_GATED_OP_FWD:
        check_forward(inputs(m, k, f, 31), kind, save=f < 10000, gap=gap)
    elif op == axo.AXO_GATED_OP_DGRAD_ACT:
        check_dgrad_act(back_inputs(m, f, k, 32), kind, gap)
    else:
        check_products(m, k, f, 33, gap)


def test_forward_no_reduction():
    """Kl = 0: act(bg) * bu."""
    d = inputs(5, 0, 40, 1)
    h, g, u = forward(d, 0)
    want = ob.gate(np.broadcast_to(d["bg"], (5, 40)), 0)[0] * d["bu"]
    bu.within(h, want, bu.BF16 * np.abs(want) + 4e-6)
    assert np.array_equal(g, np.broadcast_to(d["bg"], (5, 40))) and np.array_equal(u, np.broadcast_to(d["bu"], (5, 40)))


def test_biases_on_the_first_shard_of_the_reduction_alone():
    d = inputs(40, 64, 48, 2)
    for ix in (0, 1):
        check_forward(d, 0, p=bu.problem(40, 128, 48, (2, 1, 1), (ix, 0, 0)), with_bias=ix == 0)


def test_columns_of_one_buffer():
    """Wg | Wu, G | U and dG | dU as column blocks of one matrix each."""
    m, k, f = 70, 96, 64
    d = inputs(m, k, f, 3)
    W, Z, H = bu.Mat(np.concatenate([d["wg"], d["wu"]], 1)), bu.Out(m, 2 * f), bu.Out(m, f)
    X = bu.Mat(d["x"])
    p, q = bu.problem(m, k, f), bu.problem(m, f, k)
    ws, n = workspace(p)
    axo.axo_gated_fwd(p, X.ptr, X.ld, W.ptr, W.ptr + 2 * f, W.ld, None, None, 0, Z.ptr, Z.ptr + 2 * f, Z.ld, H.ptr, H.ld, ws.data_ptr(), n, bu.stream())
    h, g, u = ob.gated_fwd(d["x"], d["wg"], d["wu"], 0)
    bounds = bu.gated_fwd_bounds(d["x"], d["wg"], d["wu"], g, u, ob.gate(g, 0)[0])
    z = Z.result()
    bu.within(H.result(), h, bounds[0])
    bu.within(z[:, :f], g, bounds[1])
    bu.within(z[:, f:], u, bounds[2])
    dH = bu.Mat(bu.draw(np.random.default_rng(4), m, f))
    dZ, dX, dW = bu.Out(m, 2 * f), bu.Out(m, k), bu.Out(k, 2 * f)
    axo.axo_gated_dact(q, dH.ptr, dH.ld, Z.ptr, Z.ptr + 2 * f, Z.ld, 0, dZ.ptr, dZ.ptr + 2 * f, dZ.ld, bu.stream())
    axo.axo_gated_dgrad(p, dZ.ptr, dZ.ptr + 2 * f, dZ.ld, W.ptr, W.ptr + 2 * f, W.ld, dX.ptr, dX.ld, ws.data_ptr(), n, bu.stream())
    axo.axo_gated_wgrad(p, X.ptr, X.ld, dZ.ptr, dZ.ptr + 2 * f, dZ.ld, dW.ptr, dW.ptr + 2 * f, dW.ld, ws.data_ptr(), n, bu.stream())
    dz = dZ.result()
    w = np.concatenate([d["wg"], d["wu"]], 1)
    bu.within(dX.result(), dz @ w.T, bu.BF16 * np.abs(dz @ w.T) + bu.product_bound(dz, w.T))
    bu.within(dW.result(), d["x"].T @ dz, bu.BF16 * np.abs(d["x"].T @ dz) + bu.product_bound(d["x"].T, dz))


def test_nan_and_infinity_stay_in_their_rows_and_columns():
    for m, k, f in ((3, 100, 40), (40, 136, 72), (300, 70, 200), (1, 1000, 64)):
        d = inputs(m, k, f, 5)
        clean = forward(d, 0)
        d["x"][m // 2, 1], d["wg"][3, f // 3] = np.nan, np.inf
        for a, c, name in zip(forward(d, 0), clean, "HGU"):
            bad = np.zeros((m, f), bool)
            bad[m // 2] = True
            assert np.isnan(a[m // 2]).all(), name
            if name != "U":
                bad[:, f // 3] = True
                assert not np.isfinite(a[:, f // 3]).any() or name == "H"  # act(-inf) is a limit or NaN, act(inf) infinite
            assert np.array_equal(a[~bad], c[~bad]), name


@pytest.mark.parametrize("kind", [0, 1, 2])
@pytest.mark.parametrize("m,f", [(1, 1), (1, 8), (3, 7), (2, 1000), (33, 65), (700, 130), (5, 4096)])
def test_element_wise_forms(m, f, kind):
    rng = np.random.default_rng(m + f)
    g, u, dh = bu.draw(rng, m, f, 3.0), bu.draw(rng, m, f), bu.draw(rng, m, f)
    G, U, dH = bu.Mat(g, 8), bu.Mat(u, 8), bu.Mat(dh)
    H, dG, dU = bu.Out(m, f), bu.Out(m, f, 16), bu.Out(m, f, 16)
    p = bu.problem(m, f, 8)
    axo.axo_gated_act(p, G.ptr, U.ptr, G.ld, kind, H.ptr, H.ld, bu.stream())
    axo.axo_gated_dact(p, dH.ptr, dH.ld, G.ptr, U.ptr, G.ld, kind, dG.ptr, dU.ptr, dG.ld, bu.stream())
    value, slope = ob.gate(g, kind)
    bu.within(H.result(), value * u, bu.BF16 * np.abs(value * u) + np.abs(u) * bu.ACT * np.maximum(1, np.abs(g)))
    want, bounds = ob.gated_dact(dh, g, u, kind), bu.gated_dact_bounds(0.0, dh, g, u, value, slope)
    bu.within(dG.result(), want[0], bounds[0])
    bu.within(dU.result(), want[1], bounds[1])


@pytest.mark.parametrize("kind", [0, 1, 2])
def test_activations_over_all_values(kind):
    """Every finite bf16 value of G below 2^120: the result is the 64-bit one rounded once, up to the arithmetic's own error."""
    bits = np.arange(1 << 16, dtype=np.uint32) << 16
    with np.errstate(invalid="ignore"):
        g = bits.view(np.float32).astype(np.float64)
    g = g[np.isfinite(g) & (np.abs(g) < 2.0 ** 120)]
    g = np.sort(g[: g.size // 8 * 8]).reshape(-1, 8)
    one = np.ones_like(g)
    G, U, H, dG, dU = bu.Mat(g), bu.Mat(one), bu.Out(*g.shape), bu.Out(*g.shape), bu.Out(*g.shape)
    p = bu.problem(g.shape[0], 8, 8)
    axo.axo_gated_act(p, G.ptr, U.ptr, G.ld, kind, H.ptr, H.ld, bu.stream())
    axo.axo_gated_dact(p, U.ptr, U.ld, G.ptr, U.ptr, G.ld, kind, dG.ptr, dU.ptr, dG.ld, bu.stream())
    with np.errstate(over="ignore", invalid="ignore"):
        far = np.clip(g, -40.0, 40.0) if kind else np.clip(g, -700.0, 700.0)
        value, slope = ob.gate(far, kind)
        value = np.where(g > far, g, np.where(g < far, 0.0, value))
    # relative error of the far tail: exp2 of an argument of up to 128 in magnitude
    bound = bu.BF16 * np.abs(value) + 4e-5 * np.abs(value) + bu.ACT * np.minimum(1.0, np.abs(g)) * 0.25 + 1e-30
    h = H.result()
    bu.within(h, value, bound)
    assert np.array_equal(h, dU.result())
    bu.within(dG.result(), slope, bu.BF16 * np.abs(slope) + bu.ACT)


def back_inputs(m, f, n, seed):
    """Of the layer behind the block: f in-features, n out-features."""
    rng = np.random.default_rng(seed)
    return {"dy": bu.draw(rng, m, n), "w": bu.draw(rng, f, n, 1.0 / np.sqrt(max(n, 1))), "g": bu.draw(rng, m, f, 1.5), "u": bu.draw(rng, m, f)}


def dgrad_act(d, kind, gap=0):
    (m, f), n = d["g"].shape, d["dy"].shape[1]
    p = bu.problem(m, f, n)
    dY, W, G, U = bu.Mat(d["dy"], gap), bu.Mat(d["w"], gap), bu.Mat(d["g"], gap + 8), bu.Mat(d["u"], gap + 8)
    dG, dU = bu.Out(m, f, gap), bu.Out(m, f, gap)
    ws, size = workspace(p)
    axo.axo_gated_dgrad_act(p, dY.ptr, dY.ld, W.ptr, W.ld, G.ptr, U.ptr, G.ld, kind, dG.ptr, dU.ptr, dG.ld, ws.data_ptr(), size, bu.stream())
    torch.cuda.synchronize()
    return dG.result(), dU.result()


def check_dgrad_act(d, kind, gap=0):
    got = dgrad_act(d, kind, gap)
    dh = d["dy"] @ d["w"].T
    value, slope = ob.gate(d["g"], kind)
    bounds = bu.gated_dact_bounds(bu.product_bound(d["dy"], d["w"].T), dh, d["g"], d["u"], value, slope)
    for a, want, bound, name in zip(got, ob.gated_dact(dh, d["g"], d["u"], kind), bounds, ("dG", "dU")):
        bu.within(a, want, bound, name)


@pytest.mark.parametrize("m,k,f", SIZES)
def test_dgrad_act(m, k, f):
    d = back_inputs(m, f, k, 3 * m + 5 * k + f)
    for kind in range(3):
        check_dgrad_act(d, kind, (0, 8, 56)[(kind + m) % 3])


@pytest.mark.parametrize("m,k,f", WHOLE)
def test_dgrad_act_whole_tiles(m, k, f):
    for kind in range(3):
        check_dgrad_act(back_inputs(m, f, k, kind), kind)


def test_dgrad_act_no_reduction():
    dg, du = dgrad_act(back_inputs(5, 40, 0, 6), 0)
    assert not dg.any() and not du.any()


def check_products(m, k, f, seed, gap=0):
    rng = np.random.default_rng(seed)
    d = inputs(m, k, f, seed)
    dg, du = bu.draw(rng, m, f), bu.draw(rng, m, f, 0.5)
    p = bu.problem(m, k, f)
    X, Wg, Wu, dG, dU = bu.Mat(d["x"], gap), bu.Mat(d["wg"], gap), bu.Mat(d["wu"], gap), bu.Mat(dg, gap + 8), bu.Mat(du, gap + 8)
    dX, dWg, dWu = bu.Out(m, k, gap), bu.Out(k, f, gap), bu.Out(k, f, gap)
    acc = [bu.Mat(bu.draw(rng, k, f, 3.0, wide=True), gap, wide=True) for _ in range(2)]
    was = [a.numpy() for a in acc]
    ws, n = workspace(p)
    st = bu.stream()
    axo.axo_gated_dgrad(p, dG.ptr, dU.ptr, dG.ld, Wg.ptr, Wu.ptr, Wg.ld, dX.ptr, dX.ld, ws.data_ptr(), n, st)
    axo.axo_gated_wgrad(p, X.ptr, X.ld, dG.ptr, dU.ptr, dG.ld, dWg.ptr, dWu.ptr, dWg.ld, ws.data_ptr(), n, st)
    axo.axo_gated_wgrad_acc(p, X.ptr, X.ld, dG.ptr, dU.ptr, dG.ld, acc[0].ptr, acc[1].ptr, acc[0].ld, ws.data_ptr(), n, st)
    torch.cuda.synchronize()
    want = ob.gated_dgrad(dg, du, d["wg"], d["wu"])
    both, ww = np.concatenate([dg, du], 1), np.concatenate([d["wg"], d["wu"]], 1)
    bu.within(dX.result(), want, bu.BF16 * np.abs(want) + bu.product_bound(both, ww.T) + 1e-38, "dX")
    for out, a, before, z, name in ((dWg, acc[0], was[0], dg, "g"), (dWu, acc[1], was[1], du, "u")):
        want, err = d["x"].T @ z, bu.product_bound(d["x"].T, z) + 1e-38
        bu.within(out.result(), want, bu.BF16 * np.abs(want) + err, "dW" + name)
        bu.within(a.numpy(), before + want, err + 2 * bu.FP32 * np.abs(before + want), "dW32" + name)
    return p, X, dG, dU, dWg, dWu


@pytest.mark.parametrize("m,k,f", SIZES)
def test_products(m, k, f):
    check_products(m, k, f, m + k + f)
    check_products(m, k, f, m + k + f + 1, 8)


@pytest.mark.parametrize("m,k,f", [(512, 2304, 192), (2100, 2200, 136), (4099, 1030, 128), (4100, 1030, 200), (600, 520, 1100)])
def test_products_whole_tiles(m, k, f):
    p, X, dG, dU, dWg, dWu = check_products(m, k, f, 9)
    if axo.axo_gated_tiles(p, axo.AXO_GATED_OP_WGRAD)[1][2] > 1:  # workgroups share tiles: another order of the sum
        return
    for z, got in ((dG, dWg), (dU, dWu)):  # the bits of two products called on their own
        alone = bu.Out(k, f)
        axo.axo_fc_wgrad(p, X.ptr, X.ld, z.ptr, z.ld, alone.ptr, alone.ld, None, 0, bu.stream())
        assert np.array_equal(alone.result(), got.result())


def test_shared_tiles_give_the_same_bits_every_time():
    """Whatever the workspace held behind its counters."""
    m, k, f = 5784, 640, 752
    p = bu.problem(m, k, f)
    assert axo.axo_gated_tiles(p, axo.AXO_GATED_OP_WGRAD)[1][2] > 1
    rng = np.random.default_rng(34)
    X, dG, dU = (bu.Mat(bu.draw(rng, m, c)) for c in (k, f, f))
    ws, n = workspace(p)
    seen = []
    for fill in (0, 255, 0):
        ws[8192:] = fill
        out = [bu.Out(k, f) for _ in range(2)]
        axo.axo_gated_wgrad(p, X.ptr, X.ld, dG.ptr, dU.ptr, dG.ld, out[0].ptr, out[1].ptr, out[0].ld, ws.data_ptr(), n, bu.stream())
        seen.append([o.result() for o in out])
    for again in seen[1:]:
        assert all(np.array_equal(a, b) for a, b in zip(seen[0], again))


def test_dgrad_takes_what_each_product_holds():
    """Infinities behind the ends of rows and NaN in one row: the two reductions end where they should, and meet."""
    m, k, f = 40, 48, 70
    d = inputs(m, k, f, 20)
    one = np.zeros((m, f))
    one[:, -1] = 1.0
    p = bu.problem(m, k, f)
    Wg, Wu, dG, dU, dX = bu.Mat(d["wg"]), bu.Mat(d["wu"]), bu.Mat(one), bu.Mat(2 * one), bu.Out(m, k)
    for t in (Wg, Wu, dG, dU):
        t.flat[:t.rows * t.ld].view(t.rows, t.ld)[:, f:] = float("inf")
    ws, n = workspace(p)
    axo.axo_gated_dgrad(p, dG.ptr, dU.ptr, dG.ld, Wg.ptr, Wu.ptr, Wg.ld, dX.ptr, dX.ld, ws.data_ptr(), n, bu.stream())
    want = torch.from_numpy(d["wg"][:, -1] + 2 * d["wu"][:, -1]).float().bfloat16().double().numpy()
    assert np.array_equal(dX.result(), np.broadcast_to(want, (m, k)))


def test_block_against_differences():
    """The whole block's gradient along a direction, from central differences of the 64-bit forward pass."""
    m, k, f = 24, 40, 56
    d = inputs(m, k, f, 21)
    rng = np.random.default_rng(22)
    wd, dy = bu.draw(rng, f, k, f ** -0.5), bu.draw(rng, m, k)
    dirs = {n: rng.standard_normal(d[n].shape) for n in ("x", "wg", "wu")}

    for kind in range(3):
        _, g, u = forward(d, kind, bias=(False, False))
        dg, du = dgrad_act({"dy": dy, "w": wd, "g": g, "u": u}, kind)
        p = bu.problem(m, k, f)
        X, Wg, Wu, dG, dU = bu.Mat(d["x"]), bu.Mat(d["wg"]), bu.Mat(d["wu"]), bu.Mat(dg), bu.Mat(du)
        dX, dWg, dWu = bu.Out(m, k), bu.Out(k, f), bu.Out(k, f)
        ws, n = workspace(p)
        axo.axo_gated_dgrad(p, dG.ptr, dU.ptr, dG.ld, Wg.ptr, Wu.ptr, Wg.ld, dX.ptr, dX.ld, ws.data_ptr(), n, bu.stream())
        axo.axo_gated_wgrad(p, X.ptr, X.ld, dG.ptr, dU.ptr, dG.ld, dWg.ptr, dWu.ptr, dWg.ld, ws.data_ptr(), n, bu.stream())
        grads = {"x": dX.result(), "wg": dWg.result(), "wu": dWu.result()}
        for name in dirs:
            loss = lambda t: ((ob.gated_fwd(*[d[q] + (t * dirs[q] if q == name else 0) for q in ("x", "wg", "wu")], kind)[0] @ wd) * dy).sum()  # noqa: E731, B023
            slope = (loss(1e-5) - loss(-1e-5)) / 2e-5
            parts = grads[name] * dirs[name]
            # four roundings to bf16 lie between (G, U, dG or dU, the gradient), each half a step of values that add up with random signs:
            # the bound is the one that holds with none cancelling
            assert abs(parts.sum() - slope) <= 8 * bu.BF16 * np.sqrt((parts ** 2).sum()) + 4 * bu.BF16 * abs(slope), (kind, name)


def test_spans_past_4_gib():
    """Operands whose 32-bit byte offsets do not reach: rows a long way apart, any entry point."""
    m, k, f = 5, 24, 40
    ld = (1 << 28) + 8
    d = inputs(m, k, f, 23)
    rng = np.random.default_rng(24)
    big = torch.empty(8 * ld, dtype=torch.bfloat16, device=bu.DEV)
    far = lambda rows, cols: big.as_strided((rows, cols), (ld, 1))  # noqa: E731
    p, q = bu.problem(m, k, f), bu.problem(m, f, k)
    ws, n = workspace(p)
    far(m, k).copy_(torch.from_numpy(d["x"]))
    Wg, Wu, H = bu.Mat(d["wg"]), bu.Mat(d["wu"]), bu.Out(m, f)
    axo.axo_gated_fwd(p, big.data_ptr(), ld, Wg.ptr, Wu.ptr, Wg.ld, None, None, 2, None, None, 0, H.ptr, H.ld, ws.data_ptr(), n, bu.stream())
    h, g, u = ob.gated_fwd(d["x"], d["wg"], d["wu"], 2)
    bu.within(H.result(), h, bu.gated_fwd_bounds(d["x"], d["wg"], d["wu"], g, u, ob.gate(g, 2)[0])[0])
    dy, wd, gz, uz = bu.draw(rng, m, k), bu.draw(rng, f, k, k ** -0.5), bu.draw(rng, m, f), bu.draw(rng, m, f)
    far(m, k).copy_(torch.from_numpy(dy))
    Wd, G, U, dG, dU = bu.Mat(wd), bu.Mat(gz), bu.Mat(uz), bu.Out(m, f), bu.Out(m, f)
    axo.axo_gated_dgrad_act(q, big.data_ptr(), ld, Wd.ptr, Wd.ld, G.ptr, U.ptr, G.ld, 1, dG.ptr, dU.ptr, dG.ld, ws.data_ptr(), n, bu.stream())
    dh, (value, slope) = dy @ wd.T, ob.gate(gz, 1)
    bounds = bu.gated_dact_bounds(bu.product_bound(dy, wd.T), dh, gz, uz, value, slope)
    bu.within(dG.result(), dh * uz * slope, bounds[0])
    bu.within(dU.result(), dh * value, bounds[1])
    far(m, f).copy_(torch.from_numpy(gz))
    other = torch.empty(8 * ld, dtype=torch.bfloat16, device=bu.DEV)
    other.as_strided((m, f), (ld, 1)).copy_(torch.from_numpy(uz))
    dX = bu.Out(m, k)
    axo.axo_gated_dgrad(p, big.data_ptr(), other.data_ptr(), ld, Wg.ptr, Wu.ptr, Wg.ld, dX.ptr, dX.ld, ws.data_ptr(), n, bu.stream())
    both, ww = np.concatenate([gz, uz], 1), np.concatenate([d["wg"], d["wu"]], 1)
    bu.within(dX.result(), both @ ww.T, bu.BF16 * np.abs(both @ ww.T) + bu.product_bound(both, ww.T))


@pytest.mark.parametrize("m,k,f", [(1, 2048, 512), (24, 520, 200), (300, 256, 640), (4701, 64, 120), (408, 2880, 8), (112, 704, 4720)])
def test_same_bits_on_any_stream_and_in_graphs(m, k, f):
    d, b = inputs(m, k, f, 25), back_inputs(m, f, k, 26)
    first = forward(d, 0) + dgrad_act(b, 0)
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        again = forward(d, 0) + dgrad_act(b, 0)
    assert all(np.array_equal(a, c) for a, c in zip(first, again))
    p, q = bu.problem(m, k, f), bu.problem(m, f, k)
    X, Wg, Wu, dY, Wd = bu.Mat(d["x"]), bu.Mat(d["wg"]), bu.Mat(d["wu"]), bu.Mat(b["dy"]), bu.Mat(b["w"])
    outs = [bu.Out(m, f) for _ in range(5)] + [bu.Out(m, k), bu.Out(k, f), bu.Out(k, f)]
    H, G, U, dG, dU, dX, dWg, dWu = outs
    (ws, n), (ws2, n2) = workspace(p), workspace(q)

    def block():
        st = bu.stream()
        axo.axo_gated_fwd(p, X.ptr, X.ld, Wg.ptr, Wu.ptr, Wg.ld, None, None, 0, G.ptr, U.ptr, G.ld, H.ptr, H.ld, ws.data_ptr(), n, st)
        axo.axo_gated_dgrad_act(q, dY.ptr, dY.ld, Wd.ptr, Wd.ld, G.ptr, U.ptr, G.ld, 0, dG.ptr, dU.ptr, dG.ld, ws2.data_ptr(), n2, st)
        axo.axo_gated_dgrad(p, dG.ptr, dU.ptr, dG.ld, Wg.ptr, Wu.ptr, Wg.ld, dX.ptr, dX.ld, ws.data_ptr(), n, st)
        axo.axo_gated_wgrad(p, X.ptr, X.ld, dG.ptr, dU.ptr, dG.ld, dWg.ptr, dWu.ptr, dWg.ld, ws.data_ptr(), n, st)

    block()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        block()
    for turn in range(3):
        X.view().copy_(torch.from_numpy(np.roll(d["x"], turn, axis=1)).bfloat16())
        block()
        torch.cuda.synchronize()
        eager = [t.view().clone() for t in outs]
        for t in outs:
            t.flat.fill_(float("nan"))
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, t.view()) for a, t in zip(eager, outs)), turn


def test_calls_share_a_workspace():
    """Calls of several shapes, cut into different numbers of slices, one behind the other on one workspace: each gets what it gets on its own."""
    shapes = [(1, 4096, 192), (2, 5120, 1336), (1, 9, 961), (40, 2104, 64), (1, 4095, 1566), (1, 2048, 8), (272, 10, 962), (408, 2880, 8), (112, 704, 4720)]
    shared = [axo.axo_gated_tiles(bu.problem(m, k, f), op)[1][2] > 1 for m, k, f in shapes for op in (0, 2)]
    assert sum(shared) >= 6
    cases, need = [], 0
    for m, k, f in shapes:
        d, p = inputs(m, k, f, m + k), bu.problem(m, k, f)
        rng = np.random.default_rng(k)
        dz = bu.draw(rng, m, f), bu.draw(rng, m, f)
        t = [bu.Mat(a) for a in (d["x"], d["wg"], d["wu"], *dz)]
        need = max(need, axo.axo_gated_workspace_bytes(p))
        cases.append((p, t, (m, k, f)))

    def run(p, t, size, ws, n):
        X, Wg, Wu, dG, dU = t
        H, dX = bu.Out(size[0], size[2]), bu.Out(size[0], size[1])
        axo.axo_gated_fwd(p, X.ptr, X.ld, Wg.ptr, Wu.ptr, Wg.ld, None, None, 0, None, None, 0, H.ptr, H.ld, ws.data_ptr(), n, bu.stream())
        axo.axo_gated_dgrad(p, dG.ptr, dU.ptr, dG.ld, Wg.ptr, Wu.ptr, Wg.ld, dX.ptr, dX.ld, ws.data_ptr(), n, bu.stream())
        return H, dX

    alone = [run(*c, *workspace(c[0])) for c in cases]
    ws = torch.zeros(need, dtype=torch.uint8, device=bu.DEV)
    for turn in range(3):
        for c, want in zip(cases[::-1] if turn % 2 else cases, alone[::-1] if turn % 2 else alone):
            got = run(*c, ws, need)
            assert all(np.array_equal(a.result(), b.result()) for a, b in zip(got, want)), (turn, c[2])


def test_more_rows_than_small_tiles_of_a_launch():
    """4.2 million rows, whose 64 x 64 tiles are more than a launch takes.  The rows repeat every 1024, which is whole tiles, so the results do, bit for bit."""
    m, k, f, period = 4200000, 64, 4096, 1024
    d, p = inputs(period, k, f, 41), bu.problem(m, k, f)
    assert axo.axo_gated_tiles(p, axo.AXO_GATED_OP_FWD)[1] == (256, 128, 1)
    X = bu.vec(d["x"]).repeat(m // period + 1, 1)[:m]
    Wg, Wu = bu.Mat(d["wg"]), bu.Mat(d["wu"])
    H = torch.full((m, f), float("nan"), dtype=torch.bfloat16, device=bu.DEV)
    ws, n = workspace(p)
    axo.axo_gated_fwd(p, X.data_ptr(), k, Wg.ptr, Wu.ptr, Wg.ld, None, None, 0, None, None, 0, H.data_ptr(), f, ws.data_ptr(), n, bu.stream())
    h, g, u = ob.gated_fwd(d["x"], d["wg"], d["wu"], 0)
    bu.within(H[:period].double().cpu().numpy(), h, bu.gated_fwd_bounds(d["x"], d["wg"], d["wu"], g, u, ob.gate(g, 0)[0])[0])
    first = H[:period].view(torch.int16)
    for at in range(0, m, 256 * period):
        some = H[at:at + 256 * period].view(torch.int16)
        whole = some.shape[0] // period * period
        assert torch.equal(some[:whole].view(-1, period, f), first.expand(whole // period, period, f)), at
        assert torch.equal(some[whole:], first[:some.shape[0] - whole]), at


@pytest.mark.parametrize("m,k,f", [(300, 100, 200), (129, 33, 130)])
def test_spans_past_4_gib_over_several_workgroups(m, k, f):
    """Every matrix in rows 16 MB apart: the general kernel on outputs of several ragged tiles, reductions of several turns, G and U kept, biases."""
    gap = (1 << 23) + 8
    check_forward(inputs(m, k, f, 42), 0, True, (True, True), gap)
    check_forward(inputs(m, k, f, 43), 2, False, (False, True), gap)
    check_dgrad_act(back_inputs(m, f, k, 44), 1, gap)
    check_products(m, k, f, 45, gap)


def test_weight_gradients_of_spans_past_4_gib():
    """Sizes whose tiles are cut into slices, with operands that the slices' 32-bit offsets do not reach: X, dG and dU, or X alone."""
    m, k, f = 4701, 64, 120
    p = bu.problem(m, k, f)
    assert axo.axo_gated_tiles(p, axo.AXO_GATED_OP_WGRAD)[1][2] > 1
    rng = np.random.default_rng(46)
    d = [bu.draw(rng, m, c) for c in (k, f, f)]
    for gaps in ((1 << 19, 1 << 19), (1 << 19, 0), (0, 1 << 19)):
        X, dG, dU = (bu.Mat(a, g) for a, g in zip(d, (gaps[0], gaps[1], gaps[1])))
        dWg, dWu = bu.Out(k, f), bu.Out(k, f)
        acc = [bu.Mat(np.full((k, f), 0.5), 0, wide=True) for _ in range(2)]
        ws, n = workspace(p)
        axo.axo_gated_wgrad(p, X.ptr, X.ld, dG.ptr, dU.ptr, dG.ld, dWg.ptr, dWu.ptr, dWg.ld, ws.data_ptr(), n, bu.stream())
        axo.axo_gated_wgrad_acc(p, X.ptr, X.ld, dG.ptr, dU.ptr, dG.ld, acc[0].ptr, acc[1].ptr, acc[0].ld, ws.data_ptr(), n, bu.stream())
        for out, a, z in ((dWg, acc[0], d[1]), (dWu, acc[1], d[2])):
            want, err = d[0].T @ z, bu.product_bound(d[0].T, z)
            bu.within(out.result(), want, bu.BF16 * np.abs(want) + err)
            bu.within(a.numpy(), want + 0.5, err + 2 * bu.FP32 * np.abs(want + 0.5))


def test_hundreds_of_millions_of_columns():
    """600 million columns through the activation, on 9.4 million 64 x 64 tiles.  They repeat every 1024, and so do the results."""
    m, period, n = 3, 1024, 8
    f = period * 585938
    d, p = back_inputs(m, period, n, 47), bu.problem(m, f, n)
    assert axo.axo_gated_tiles(p, axo.AXO_GATED_OP_DGRAD_ACT)[1] == (64, 64, 1)
    dY, W = bu.vec(d["dy"]), bu.vec(d["w"]).repeat(f // period, 1)
    G, U = (bu.vec(d[c]).repeat(1, f // period) for c in "gu")
    dG, dU = (torch.full((m, f), float("nan"), dtype=torch.bfloat16, device=bu.DEV) for _ in range(2))
    ws, size = workspace(p)
    axo.axo_gated_dgrad_act(p, dY.data_ptr(), n, W.data_ptr(), n, G.data_ptr(), U.data_ptr(), f, 1, dG.data_ptr(), dU.data_ptr(), f, ws.data_ptr(), size, bu.stream())
    dh, (value, slope) = d["dy"] @ d["w"].T, ob.gate(d["g"], 1)
    bounds = bu.gated_dact_bounds(bu.product_bound(d["dy"], d["w"].T), dh, d["g"], d["u"], value, slope)
    for t, want, bound in zip((dG, dU), ob.gated_dact(dh, d["g"], d["u"], 1), bounds):
        bu.within(t[:, :period].double().cpu().numpy(), want, bound)
        bits = t.view(torch.int16).view(m, f // period, period)
        assert torch.equal(bits, bits[:, :1].expand(-1, f // period, -1))
