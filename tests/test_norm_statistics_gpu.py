"""Layer norm of rows far from zero: a mean hundreds of deviations away, where a variance from squares has no correct digits left.  The bounds are those of
the sums as the kernels form them, a few dozen additions one behind the other and a tree, and are shown to tell: the best that squares can give in fp32, and
outputs of zero, are outside at every width."""
import numpy as np
import pytest

torch = pytest.importorskip("torch")
import block_util as bu
import paper_2305_13525_amd as axo
from oracle import block as ob
from test_norm_gpu import EPS, forward, inputs

# (bf16 or fp32, mean): deviations of 1.5, and 2 and more where bf16 values lie two apart
KINDS = [(False, 256.0), (True, 1000.0)]
WIDTHS = [40, 64, 100, 250, 500, 1000, 2000, 4000, 5000, 8200, 12000, 16000, 20000, 24584, 32768, 33000, 70000]
# parts of a split width, each of so many columns
SPLITS = [(2, 48), (4, 512), (3, 1000), (2, 5000), (2, 33000), (8, 256)]


def additions(k):
    """How many additions, at most, lie between a value and its row's sum: up to 32 values of a lane (rows in registers), or all of a thread's of a row of any length (eight
    in every 8192), six steps among the lanes of a wave, and up to 16 waves one behind the other."""
    return max(32, (k + 8191) // 8192 * 8) + 6 + 16


def bounds(s, mean, rstd, gamma, beta, y, n, parts=1):
    """Bounds of y, mean and rstd where every sum is off by at most n roundings of its terms' magnitudes, and the statistics are joined from those of so many parts."""
    eps_mean = (n + 2) * bu.FP32 * np.abs(s).mean(axis=1)
    dev = np.abs(s - mean[:, None])
    # the variance around a mean that is off by eps_mean is larger by its square; each deviation is rounded, squared and added up
    rel_rstd = 0.5 * (eps_mean * rstd) ** 2 + 0.5 * (n + 8) * bu.FP32 + 4 * bu.FP32
    # the means of parts lie off the whole row's, and what each is off by (and the whole row's) counts twice in the square of that
    apart = np.abs(s.reshape(s.shape[0], parts, -1).mean(axis=2) - mean[:, None]).mean(axis=1)
    rel_rstd = rel_rstd + 2 * apart * eps_mean * rstd ** 2
    err = ((dev * (rel_rstd[:, None] + 4 * bu.FP32) + eps_mean[:, None]) * rstd[:, None]) * np.abs(gamma)
    err = err + 4 * bu.FP32 * (dev * rstd[:, None] * np.abs(gamma) + np.abs(beta))
    return bu.BF16 * (np.abs(y) + err) + err, eps_mean, rel_rstd * rstd


def far(m, k, wide, mean):
    d = inputs(m, k, wide, 50 + k, mean)
    return d, *ob.norm_fwd(d["x"], d["gamma"], d["beta"], EPS)


@pytest.mark.parametrize("wide,mean", KINDS)
@pytest.mark.parametrize("k", WIDTHS + [a * b for a, b in SPLITS])
def test_bounds_tell(k, wide, mean):
    """Squares: the mean and the mean of squares each rounded once to fp32, which no kernel's are better than."""
    d, y, m, r = far(4, k, wide, mean)
    by, bm, br = bounds(d["x"], m, r, d["gamma"], d["beta"], y, additions(k) + 8)
    m32 = m.astype(np.float32)
    var = np.maximum((d["x"] ** 2).mean(axis=1).astype(np.float32) - m32 * m32, np.float32(0.0)).astype(np.float64)
    naive = 1.0 / np.sqrt(var + EPS)
    assert np.any(np.abs(naive - r) > br)
    from_squares = (d["x"] - m[:, None]) * naive[:, None] * d["gamma"] + d["beta"]
    assert np.all(np.any(np.abs(y) > by, axis=1))  # an output of zeros, row by row
    assert np.any(np.abs(from_squares - y) > by) or np.abs(naive / r - 1.0).max() < 2 * bu.BF16  # less than a rounding of the output


@pytest.mark.gpu
@pytest.mark.parametrize("wide,mean", KINDS)
@pytest.mark.parametrize("k", WIDTHS)
def test_far_from_zero(k, wide, mean):
    d, y, m, r = far(4, k, wide, mean)
    _, got, st = forward(d, wide, False)
    by, bm, br = bounds(d["x"], m, r, d["gamma"], d["beta"], y, additions(k))
    bu.within(st[:, 0], m, bm, "mean")
    bu.within(st[:, 1], r, br, "rstd")
    bu.within(got, y, by, "y")


@pytest.mark.gpu
@pytest.mark.parametrize("parts,kl", SPLITS)
@pytest.mark.parametrize("wide,mean", KINDS)
def test_far_from_zero_in_halves(parts, kl, wide, mean):
    """The statistics of the shards of a split width, joined: the shards' own deviations and those of their means."""
    m, k = 4, parts * kl
    d, y, mean64, r = far(m, k, wide, mean)
    X, Y, st = bu.Mat(d["x"], 0, wide), bu.Out(m, k), torch.full((m, 2), float("nan"), device=bu.DEV)
    gm, bt, gathered = bu.vec(d["gamma"]), bu.vec(d["beta"]), torch.full((parts, m, 2), float("nan"), device=bu.DEV)
    shard = lambda i: bu.problem(m, k, 0, (parts, 1, 1), (i, 0, 0))  # noqa: E731
    at = lambda i, e: i * kl * e  # noqa: E731
    e = 4 if wide else 2
    for i in range(parts):
        axo.axo_norm_part(shard(i), X.ptr + at(i, e), X.ld, None, 0, int(wide), None, 0, gathered[i].data_ptr(), bu.stream())
    for i in range(parts):
        axo.axo_norm_apply(shard(i), X.ptr + at(i, e), X.ld, int(wide), gathered.data_ptr(), parts, gm.data_ptr() + at(i, 2), bt.data_ptr() + at(i, 2), EPS,
                           Y.ptr + at(i, 2), Y.ld, st.data_ptr(), bu.stream())
    torch.cuda.synchronize()
    by, bm, br = bounds(d["x"], mean64, r, d["gamma"], d["beta"], y, additions(kl) + parts, parts)
    got = st.double().cpu().numpy()
    bu.within(got[:, 0], mean64, bm, "mean")
    bu.within(got[:, 1], r, br, "rstd")
    bu.within(Y.result(), y, by, "y")


@pytest.mark.gpu
@pytest.mark.parametrize("transposed", [0, 1])
@pytest.mark.parametrize("k,parts", [(96, 2), (2048, 4), (3000, 3), (24, 1), (20480, 2), (66000, 2), (50000, 2)])
def test_split_width_in_fp32(k, parts, transposed):
    """An fp32 stream in halves, forward with a residual and backward with its gradient, in place in the whole matrices, joined on the test's side."""
    m, kl = 9, k // parts
    d = inputs(m, k, True, 16)
    s = torch.from_numpy(d["x"] + d["r"]).float().double().numpy()
    X, R, dY, dR = bu.Mat(d["x"], 0, True), bu.Mat(d["r"], 8, True), bu.Mat(d["dy"]), bu.Mat(d["r"], 0, True)
    S, Y, dX = bu.Out(m, k, 0, True), bu.Out(m, k), bu.Out(m, k, 16, True)
    gm, bt = bu.vec(d["gamma"]), bu.vec(d["beta"])
    st, gathered = torch.full((m, 2), float("nan"), device=bu.DEV), torch.full((parts, m, 2), float("nan"), device=bu.DEV)
    grid = (1, parts, 1) if transposed else (parts, 1, 1)
    shard = lambda i: bu.problem(m, k, 0, grid, (0, i, 0) if transposed else (i, 0, 0), transposed)  # noqa: E731
    for i in range(parts):
        axo.axo_norm_part(shard(i), X.ptr + 4 * i * kl, X.ld, R.ptr + 4 * i * kl, R.ld, 1, S.ptr + 4 * i * kl, S.ld, gathered[i].data_ptr(), bu.stream())
    for i in range(parts):
        axo.axo_norm_apply(shard(i), S.ptr + 4 * i * kl, S.ld, 1, gathered.data_ptr(), parts, gm.data_ptr() + 2 * i * kl, bt.data_ptr() + 2 * i * kl, EPS,
                           Y.ptr + 2 * i * kl, Y.ld, st.data_ptr(), bu.stream())
    torch.cuda.synchronize()
    assert np.array_equal(S.result(), s)
    y, mean, rstd = ob.norm_fwd(s, d["gamma"], d["beta"], EPS)
    by, bm, br = bounds(s, mean, rstd, d["gamma"], d["beta"], y, additions(kl) + parts, parts)
    got = st.double().cpu().numpy()
    bu.within(got[:, 0], mean, bm, "mean")
    bu.within(got[:, 1], rstd, br, "rstd")
    bu.within(Y.result(), y, by, "y")

    sums = torch.full((parts, m, 2), float("nan"), device=bu.DEV)
    dg, db = torch.full((k,), float("nan"), device=bu.DEV), torch.full((k,), float("nan"), device=bu.DEV)
    for i in range(parts):
        n = axo.axo_norm_workspace_bytes(shard(i))
        ws = torch.full((max(n, 16),), 255, dtype=torch.uint8, device=bu.DEV)
        axo.axo_norm_bwd_part(shard(i), dY.ptr + 2 * i * kl, dY.ld, S.ptr + 4 * i * kl, S.ld, 1, gm.data_ptr() + 2 * i * kl, st.data_ptr(), sums[i].data_ptr(),
                              dg.data_ptr() + 4 * i * kl, db.data_ptr() + 4 * i * kl, 0, ws.data_ptr(), n, bu.stream())
    total = sums.sum(0)
    for i in range(parts):
        axo.axo_norm_bwd_apply(shard(i), dY.ptr + 2 * i * kl, dY.ld, S.ptr + 4 * i * kl, S.ld, dR.ptr + 4 * i * kl, dR.ld, 1, gm.data_ptr() + 2 * i * kl, st.data_ptr(),
                               total.data_ptr(), dX.ptr + 4 * i * kl, dX.ld, bu.stream())
    torch.cuda.synchronize()
    want = ob.norm_bwd(d["dy"], s, got[:, 0], got[:, 1], d["gamma"], d["r"])
    limits = bu.norm_bwd_bounds(d["dy"], s, got[:, 0], got[:, 1], d["gamma"], d["r"], want[0], True)
    bu.within(dX.result(), want[0], limits[0], "dx")
    bu.within(dg.double().cpu().numpy(), want[1], limits[1], "dgamma")
    bu.within(db.double().cpu().numpy(), want[2], limits[2], "dbeta")
