"""The gated block on inputs whose rows start anywhere in a cache line.  Forward and through the activation, every kind of tiles of gemm_tile.hpp fetches such
rows by whole lines where the reduction is long enough; where the rows lie must not show in the results, which are compared bit for bit with
those of the same values in rows that start on lines, and these with 64-bit products.  Everything around the inputs is NaN.  The same for outputs: in
rows that straddle lines, which are stored plainly, or, forward and past 128 MB, past the caches."""
import numpy as np
import pytest
import torch

import block_util as bu
import paper_2305_13525_amd as axo
from oracle import block as ob
from test_gated_gpu import workspace
from test_line_loads_gpu import kinds, placed

pytestmark = pytest.mark.gpu

WHOLE, HALF, MIXED = axo.AXO_KERNEL_TILES_256, axo.AXO_KERNEL_TILES_256_HALF, axo.AXO_KERNEL_TILES_256_MIXED
FWD, DACT = axo.AXO_GATED_OP_FWD, axo.AXO_GATED_OP_DGRAD_ACT

# tokens, reduction, width of the outputs; rows and columns of the tiles; of 256-row ones, whether all are whole, half as wide or some of each.  Reductions of
# every remainder of the rings, with ends inside a step, a chunk and on them, and the shortest that lines are taken for
FORWARD = [
    (260, 768, 61, 64, 32, 0), (261, 903, 62, 64, 32, 0), (259, 1025, 63, 64, 32, 0), (2241, 1408, 60, 64, 32, 0),
    (329, 520, 1347, 64, 64, 0), (201, 640, 2101, 64, 64, 0), (261, 1151, 1640, 64, 64, 0),
    (257, 768, 3386, 128, 64, 0), (217, 570, 4159, 128, 64, 0), (207, 903, 4204, 128, 64, 0), (204, 1025, 4469, 128, 64, 0),
    (344, 512, 8958, 256, 128, WHOLE), (518, 520, 5476, 256, 128, WHOLE), (339, 725, 8420, 256, 128, WHOLE), (327, 1151, 8267, 256, 128, WHOLE),
    (329, 520, 8217, 256, 128, MIXED), (521, 640, 5687, 256, 128, MIXED), (326, 1025, 8606, 256, 128, MIXED)]
BACK = [
    (2128, 768, 64, 64, 64, 0), (2095, 903, 60, 64, 64, 0), (2089, 1025, 62, 64, 64, 0), (2241, 1408, 60, 64, 64, 0),
    (330, 640, 2715, 64, 128, 0), (258, 830, 3421, 64, 128, 0), (200, 1151, 4199, 64, 128, 0),
    (257, 512, 6728, 128, 128, 0), (205, 570, 8631, 128, 128, 0), (267, 830, 6593, 128, 128, 0), (204, 1025, 8472, 128, 128, 0),
    (781, 512, 8354, 256, 256, WHOLE), (775, 570, 8933, 256, 256, WHOLE), (1031, 903, 6897, 256, 256, WHOLE),
    (861, 512, 7061, 256, 256, HALF), (514, 1025, 7449, 256, 256, HALF), (706, 725, 8450, 256, 256, HALF),
    (772, 512, 8471, 256, 256, MIXED), (795, 768, 8218, 256, 256, MIXED), (795, 1025, 8304, 256, 256, MIXED)]
# (chunks of 8 by which rows of A are longer than lines, chunks that the first starts behind one, the same of B)
PLACES = [(i, 0, i, 0) for i in range(1, 8)] + [(0, 3, 0, 0), (0, 7, 0, 1), (1, 7, 0, 0), (3, 2, 5, 4)]


def normal(gen, rows, cols, sigma=1.0):
    return (torch.randn(rows, cols, device=bu.DEV, generator=gen) * sigma).bfloat16()


def exact(a, b):
    """(a @ b, the bound of an fp32 sum of it) in 64 bits."""
    a, b = a.double(), b.double()
    return (a @ b).cpu().numpy(), (2 * (a.shape[1] + 4) * bu.FP32 * (a.abs() @ b.abs())).cpu().numpy()


def outputs(rows, cols, n, extra=0, shift=0):
    """n matrices of NaN, in rows `extra` chunks longer than whole lines, the first `shift` chunks behind a line."""
    return [placed(torch.full((rows, cols), float("nan"), dtype=torch.bfloat16, device=bu.DEV), extra, shift) for _ in range(n)]


def padding_untouched(t):
    """Nothing was written between the rows, ahead of the first or behind the last one."""
    rows, cols = t.shape
    flat = torch.as_strided(t, (t.untyped_storage().nbytes() // 2,), (1,), 0)
    between = torch.as_strided(t, (rows, t.stride(0) - cols), (t.stride(0), 1), t.storage_offset() + cols)
    return bool(between.isnan().all()) and bool(flat[:t.storage_offset()].isnan().all())


def forward(p, x, wg, wu, bg, bv, out, kind, save=True):
    ws, n = workspace(p)
    h, g, u = out
    axo.axo_gated_fwd(p, x.data_ptr(), x.stride(0), wg.data_ptr(), wu.data_ptr(), wg.stride(0), bg.data_ptr(), bv.data_ptr(), kind, g.data_ptr() if save else None,
                      u.data_ptr() if save else None, g.stride(0) if save else 0, h.data_ptr(), h.stride(0), ws.data_ptr(), n, bu.stream())
    torch.cuda.synchronize()
    assert all(padding_untouched(t) for t in out)
    return [t.clone().view(torch.int16) for t in (out if save else out[:1])]


def check_forward(got, x, wg, wu, bg, bv, kind):
    (g, eg), (u, eu) = exact(x, wg), exact(x, wu)
    g, u = g + bg.double().cpu().numpy(), u + bv.double().cpu().numpy()
    eg, eu = eg + 2 * bu.FP32 * np.abs(g), eu + 2 * bu.FP32 * np.abs(u)
    value = ob.gate(g, kind)[0]
    bound = bu.BF16 * np.abs(value * u) + np.abs(u) * (bu.SLOPE * eg + bu.ACT * np.maximum(1.0, np.abs(g))) + np.abs(value) * eu + bu.SLOPE * eg * eu
    for t, want, b, name in zip(got, (value * u, g, u), (bound, bu.BF16 * np.abs(g) + eg, bu.BF16 * np.abs(u) + eu), "HGU"):
        bu.within(t.view(torch.bfloat16).double().cpu().numpy(), want, b + 1e-38, name)


@pytest.mark.parametrize("m,k,f,rows,cols,large", FORWARD)
def test_forward(m, k, f, rows, cols, large):
    gen = torch.Generator(device=bu.DEV)
    gen.manual_seed(m + k + f)
    x, wg, wu, bg, bv = normal(gen, m, k), normal(gen, k, f, 1.5 * k ** -0.5), normal(gen, k, f, 1.5 * k ** -0.5), normal(gen, 1, f)[0], normal(gen, 1, f)[0]
    p, both = bu.problem(m, k, f), bu.problem(m, k, 2 * f)
    assert axo.axo_gated_tiles(p, FWD)[1] == (rows, cols, 1)
    kind = f % 2

    def run(place):
        X, (Wg, Wu) = placed(x, *place[:2]), (placed(w, *place[2:]) for w in (wg, wu))
        if large:  # the tiles of a product of both projections' columns
            ld = 2 * Wg.stride(0)
            tiles = axo.axo_fc_tiles(both, axo.AXO_OP_FWD, X.data_ptr(), X.stride(0), Wg.data_ptr(), ld, ld)[1]
            assert axo.axo_fc_kernel(both, axo.AXO_OP_FWD, X.stride(0), ld, ld)[1] == large
            assert kinds(tiles >> 16) == ({WHOLE} if place[:2] != (0, 0) else set()), place
        return forward(p, X, Wg, Wu, bg, bv, outputs(m, f, 3), kind)

    want = run((0, 0, 0, 0))
    check_forward(want, x, wg, wu, bg, bv, kind)
    for place in [q for q in PLACES if q[0] != 4]:  # with half of its rows straddling a product takes lines from 24 steps on
        assert all(torch.equal(a, b) for a, b in zip(run(place), want)), place


@pytest.mark.parametrize("m,k,f,rows,cols,large", BACK)
def test_through_the_activation(m, k, f, rows, cols, large):
    gen = torch.Generator(device=bu.DEV)
    gen.manual_seed(m + k + f)
    dy, w, g, u = normal(gen, m, k), normal(gen, f, k, k ** -0.5), normal(gen, m, f, 1.5), normal(gen, m, f)
    p = bu.problem(m, f, k)
    assert axo.axo_gated_tiles(p, DACT)[1] == (rows, cols, 1)
    kind, ws = f % 2, workspace(p)

    def run(place):
        dY, W, G, U = placed(dy, *place[:2]), placed(w, *place[2:]), placed(g, *place[2:]), placed(u, *place[2:])
        if large:
            tiles = axo.axo_fc_tiles(p, axo.AXO_OP_DGRAD, dY.data_ptr(), dY.stride(0), W.data_ptr(), W.stride(0), (f + 63) // 64 * 64)[1]
            assert axo.axo_fc_kernel(p, axo.AXO_OP_DGRAD, dY.stride(0), W.stride(0), (f + 63) // 64 * 64)[1] == large
            every = {WHOLE, HALF} if large == MIXED else {large}
            if place == (0, 0, 0, 0): every = set()
            elif place[2:] == (0, 0): every -= {HALF}  # rows of dY alone are less than two thirds of a half-width step's
            assert kinds(tiles >> 16) == every, place
        dG, dU = outputs(m, f, 2)
        axo.axo_gated_dgrad_act(p, dY.data_ptr(), dY.stride(0), W.data_ptr(), W.stride(0), G.data_ptr(), U.data_ptr(), G.stride(0), kind, dG.data_ptr(), dU.data_ptr(),
                                dG.stride(0), ws[0].data_ptr(), ws[1], bu.stream())
        torch.cuda.synchronize()
        assert padding_untouched(dG) and padding_untouched(dU)
        return [t.clone().view(torch.int16) for t in (dG, dU)]

    want = run((0, 0, 0, 0))
    dh, err = exact(dy, w.t())
    gd, ud = g.double().cpu().numpy(), u.double().cpu().numpy()
    bounds = bu.gated_dact_bounds(err, dh, gd, ud, *ob.gate(gd, kind))
    for t, full, bound, name in zip(want, ob.gated_dact(dh, gd, ud, kind), bounds, ("dG", "dU")):
        bu.within(t.view(torch.bfloat16).double().cpu().numpy(), full, bound, name)
    for place in [q for q in PLACES if q[0] != 4]:
        assert all(torch.equal(a, b) for a, b in zip(run(place), want)), place


# H, G and U of 138 to 140 MB, and H alone of that; with a reduction that rows by lines are taken for, and without
@pytest.mark.parametrize("m,k,f,rows,cols,save", [
    (2112, 64, 11000, 256, 128, True), (2112, 520, 11000, 256, 128, True), (2100, 520, 11003, 256, 128, True), (16640, 64, 4200, 256, 128, False),
    (2799, 8, 8333, 256, 128, True)])
def test_outputs_past_the_caches(m, k, f, rows, cols, save):
    gen = torch.Generator(device=bu.DEV)
    gen.manual_seed(f)
    x, wg, wu, bg, bv = normal(gen, m, k), normal(gen, k, f, 1.5 * k ** -0.5), normal(gen, k, f, 1.5 * k ** -0.5), normal(gen, 1, f)[0], normal(gen, 1, f)[0]
    p = bu.problem(m, k, f)
    assert axo.axo_gated_tiles(p, FWD)[1] == (rows, cols, 1) and m * f * (6 if save else 2) > 128 << 20
    want = None
    for inputs in ((0, 0), (1, 0)):  # without and with rows by lines
        X, Wg, Wu = placed(x, *inputs), placed(wg, *inputs), placed(wu, *inputs)
        for extra, shift in ((0, 0), (1, 0), (4, 0), (7, 0), (0, 5), (3, 2)):
            got = forward(p, X, Wg, Wu, bg, bv, outputs(m, f, 3, extra, shift), 0, save)
            if want is None:
                want = got
                check_forward(want, x, wg, wu, bg, bv, 0)
            assert all(torch.equal(a, b) for a, b in zip(got, want)), (inputs, extra, shift)


@pytest.mark.parametrize("m,k,f", [(300, 64, 513), (257, 192, 320), (640, 200, 264), (130, 130, 130), (1001, 259, 515), (512, 96, 2304)])
def test_outputs_in_rows_that_straddle_lines(m, k, f):
    """Fewer: whether rows of the outputs are stored plainly or not, on the tiles that these sizes take."""
    gen = torch.Generator(device=bu.DEV)
    gen.manual_seed(f)
    x, wg, wu, bg, bv = normal(gen, m, k), normal(gen, k, f, 1.5 * k ** -0.5), normal(gen, k, f, 1.5 * k ** -0.5), normal(gen, 1, f)[0], normal(gen, 1, f)[0]
    X, Wg, Wu = placed(x, 0, 0), placed(wg, 0, 0), placed(wu, 0, 0)
    want = None
    for extra, shift in ((0, 0), (1, 0), (4, 0), (0, 5), (3, 2)):
        got = forward(bu.problem(m, k, f), X, Wg, Wu, bg, bv, outputs(m, f, 3, extra, shift), 0)
        if want is None:
            want = got
            check_forward(want, x, wg, wu, bg, bv, 0)
        assert all(torch.equal(a, b) for a, b in zip(got, want)), (extra, shift)
