"""The norms either side of a residual addition on the GPU, forward and backward, against the 64-bit definition."""
import numpy as np
import pytest

torch = pytest.importorskip("torch")
import block_util as bu
import residual_util as ru
import paper_2305_13525_amd as axo
from oracle import residual as orr

pytestmark = pytest.mark.gpu
EPS, SCALE = 1e-5, 0.75
VECTORS = ("gamma_a", "beta_a", "gate", "gamma_b", "beta_b")
GRADS = ("dgamma_a", "dbeta_a", "dgate", "dgamma_b", "dbeta_b")
DEFAULT = {"gamma_a": 1.0, "beta_a": 0.0, "gate": 1.0, "gamma_b": 1.0, "beta_b": 0.0}

# rows x columns: one value, below and around a wave, a power of two either side, odd lengths, rows past what fits registers
SIZES = [(1, 1), (1, 8), (3, 7), (2, 9), (5, 33), (70, 64), (2, 65), (130, 127), (17, 128), (4, 250), (9, 256), (2, 257), (5, 512), (3, 513), (33, 1000),
         (4, 1024), (35, 1027), (2, 2048), (3, 2056), (1, 4096), (300, 4096), (2, 4099), (3, 7168), (2, 8192), (2, 9000), (3, 12288), (2, 16384),
         (2, 16385), (2, 20000), (1, 33001)]
KINDS = [(a, b) for a in (orr.NONE, orr.LAYER, orr.RMS) for b in (orr.LAYER, orr.RMS)]


def inputs(m, k, wide, seed):
    rng = np.random.default_rng(seed)
    d = {"b": bu.draw(rng, m, k, 1.5, 0.3), "x": bu.draw(rng, m, k, 2.0, 0.5, wide), "dy": bu.draw(rng, m, k), "ds": bu.draw(rng, m, k, 1.0, 0.1, wide)}
    for name in VECTORS:
        d[name] = bu.draw(rng, 1, k, 0.2, DEFAULT[name])[0]
    return d


def stored(a, wide):
    t = torch.from_numpy(a).float()
    return (t if wide else t.bfloat16()).double().numpy()


def vectors(d, without=()):
    """(pointers' tensors, 64-bit values) of the five vectors; NULL where left out."""
    dev = {n: None if n in without else bu.vec(d[n]) for n in VECTORS}
    return dev, {n: DEFAULT[n] if n in without else d[n] for n in VECTORS}


def forward(d, kinds, wide, gap=0, without=(), stats=True, eps=EPS, scale=SCALE):
    m, k = d["b"].shape
    p = bu.problem(m, k, 0)
    B, X = bu.Mat(d["b"], gap), bu.Mat(d["x"], gap + 8, wide)
    S, Y = bu.Out(m, k, gap, wide), bu.Out(m, k, gap + 16)
    st = torch.full((m, 4), float("nan"), device=bu.DEV) if stats else None
    dev, _ = vectors(d, without)
    axo.axo_resnorm_fwd(p, B.ptr, B.ld, X.ptr, X.ld, int(wide), kinds[0], bu.ptr(dev["gamma_a"]), bu.ptr(dev["beta_a"]), bu.ptr(dev["gate"]), scale, kinds[1],
                        bu.ptr(dev["gamma_b"]), bu.ptr(dev["beta_b"]), eps, S.ptr, S.ld, Y.ptr, Y.ld, bu.ptr(st), bu.stream())
    torch.cuda.synchronize()
    return S.result(), Y.result(), None if st is None else st.double().cpu().numpy()


def check_forward(d, kinds, wide, gap=0, without=(), eps=EPS, scale=SCALE):
    S, Y, st = forward(d, kinds, wide, gap, without, True, eps, scale)
    _, v = vectors(d, without)
    s, mean, rstd = orr.resnorm_s(d["b"], d["x"], scale, kinds[0], v["gamma_a"], v["beta_a"], v["gate"], eps)
    bu.within(S, s, ru.s_bound(d["b"], d["x"], scale, kinds[0], mean, rstd, v["gamma_a"], v["beta_a"], v["gate"], s, wide), "s")
    y, mean_b, rstd_b = orr.resnorm_y(S, kinds[1], v["gamma_b"], v["beta_b"], eps)  # of the stream as it is stored
    bu.within(Y, y, ru.y_bound(S, kinds[1], mean_b, rstd_b, v["gamma_b"], v["beta_b"], y), "y")
    for at, values, kind, m, r in ((0, d["b"], kinds[0], mean, rstd), (2, S, kinds[1], mean_b, rstd_b)):
        em, er, _ = ru.normed_bounds(values, kind, m, r)
        bu.within(st[:, at], m, em + 1e-38, "mean")
        bu.within(st[:, at + 1], r, er + 1e-38, "rstd")


@pytest.mark.parametrize("m,k", SIZES)
@pytest.mark.parametrize("wide", [False, True])
def test_forward(m, k, wide):
    d = inputs(m, k, wide, 100 * m + k)
    for i, kinds in enumerate(KINDS):
        check_forward(d, kinds, wide, gap=8 * (i % 2))


def test_forward_without_vectors():
    for m, k in ((3, 100), (2, 4104), (2, 17000)):
        d = inputs(m, k, False, 7)
        check_forward(d, (1, 1), False, 8, without=VECTORS)
        for name in VECTORS:
            check_forward(d, (1, 2), False, 0, without=(name,))
        assert forward(d, (2, 1), False, stats=False)[2] is None


def test_scale_and_eps():
    d = inputs(3, 200, False, 10)
    check_forward(d, (2, 2), False, eps=0.0)
    check_forward(d, (1, 1), False, eps=3.0, scale=-2.0)
    S, _, _ = forward(d, (1, 1), False, scale=0.0)
    assert np.array_equal(S, d["x"])


def test_far_from_zero():
    """A mean a thousand deviations from zero: the variance comes from deviations, not from squares."""
    for k in (64, 1000, 5000, 17000):
        d = inputs(4, k, True, 8)
        d["x"] += 1024.0
        check_forward(d, (1, 1), True)


def test_constant_rows():
    d = inputs(3, 200, False, 9)
    d["b"][:], d["x"][:] = 2.5, -1.0
    d["gate"][:], d["beta_a"][:] = 1.0, 0.5
    S, Y, st = forward(d, (1, 1), False, scale=1.0)
    assert np.array_equal(S, np.full((3, 200), -0.5)) and np.array_equal(Y, np.broadcast_to(d["beta_b"], Y.shape)) and np.array_equal(st[:, 0], [2.5] * 3)


def test_infinities_and_nans_stay_in_their_rows():
    for k in (40, 1000, 4096, 12288, 17000):
        d = inputs(6, k, False, 11)
        clean = forward(d, (1, 1), False)
        back = backward(d, (1, 1), False)[1]
        d["b"][1, k // 2], d["x"][4, 0] = np.inf, np.nan
        got = forward(d, (1, 1), False)
        for row in range(6):
            if row in (1, 4):
                assert np.isnan(got[1][row]).all()
            else:
                assert all(np.array_equal(g[row], c[row]) for g, c in zip(got, clean))
        d = inputs(6, k, False, 11)
        d["dy"][2, k - 1] = np.nan
        got = backward(d, (1, 1), False)[1]
        for row in range(6):
            if row == 2:
                assert np.isnan(got[0][row]).all() and np.isnan(got[1][row]).all()
            else:
                assert np.array_equal(got[0][row], back[0][row]) and np.array_equal(got[1][row], back[1][row])


def backward(d, kinds, wide, gap=0, without=(), which=GRADS, acc=None, ds=True, scale=SCALE):
    m, k = d["b"].shape
    _, v = vectors(d, without)
    if m and k:
        s, ma, ra = orr.resnorm_s(d["b"], d["x"], scale, kinds[0], v["gamma_a"], v["beta_a"], v["gate"], EPS)
        s = stored(s, wide)
        _, mb, rb = orr.resnorm_y(np.where(np.isfinite(s), s, 0.0), kinds[1], 1.0, 0.0, EPS)
    else:
        s, (ma, ra, mb, rb) = d["x"], [np.zeros(m)] * 4
    st = torch.from_numpy(np.stack([ma, ra, mb, rb], 1)).float().to(bu.DEV)
    p = bu.problem(m, k, 0)
    dY, dS, B, S = bu.Mat(d["dy"], gap), bu.Mat(d["ds"], gap + 8, wide) if ds else None, bu.Mat(d["b"], gap + 16), bu.Mat(s, gap, wide)
    dX, dB = bu.Out(m, k, gap + 8, wide), bu.Out(m, k, gap)
    start = np.full(k, np.nan) if acc is None else acc
    out = {n: torch.from_numpy(start).float().to(bu.DEV) if n in which else None for n in GRADS}
    dev, _ = vectors(d, without)
    n = axo.axo_resnorm_workspace_bytes(p)
    ws = torch.full((max(n, 16),), 255, dtype=torch.uint8, device=bu.DEV)
    axo.axo_resnorm_bwd(p, dY.ptr, dY.ld, bu.ptr(dS), dS.ld if ds else 0, B.ptr, B.ld, S.ptr, S.ld, int(wide), kinds[0], bu.ptr(dev["gamma_a"]), bu.ptr(dev["beta_a"]),
                        bu.ptr(dev["gate"]), scale, kinds[1], bu.ptr(dev["gamma_b"]), st.data_ptr(), dX.ptr, dX.ld, dB.ptr, dB.ld,
                        *[bu.ptr(out[g]) for g in GRADS], int(acc is not None), ws.data_ptr() if which else None, n if which else 0, bu.stream())
    torch.cuda.synchronize()
    got = [dX.result(), dB.result()] + [None if out[g] is None else out[g].double().cpu().numpy() for g in GRADS]
    return (s, st.double().cpu().numpy()), got


def check_backward(d, kinds, wide, gap=0, without=(), which=GRADS, acc=None, ds=True, scale=SCALE):
    (s, st), got = backward(d, kinds, wide, gap, without, which, acc, ds, scale)
    _, v = vectors(d, without)
    args = (d["dy"], d["ds"] if ds else None, d["b"], s, st, scale, *kinds, v["gamma_a"], v["beta_a"], v["gate"], v["gamma_b"])
    want = orr.resnorm_bwd(*args)
    bounds = ru.resnorm_bwd_bounds(*args, want, wide)
    for i, name in enumerate(("dx", "db") + GRADS):
        if got[i] is None:
            continue
        start = acc if acc is not None and i >= 2 else 0.0
        bu.within(got[i], want[i] + start, bounds[i] + 2 * bu.FP32 * np.abs(start), name)


@pytest.mark.parametrize("m,k", SIZES + [(513, 40), (1030, 100), (5000, 72), (700, 1100)])
@pytest.mark.parametrize("wide", [False, True])
def test_backward(m, k, wide):
    d = inputs(m, k, wide, 200 * m + k)
    for i, kinds in enumerate(KINDS if m * k < 100000 else KINDS[2:4]):
        check_backward(d, kinds, wide, gap=8 * (i % 2), ds=i % 3 != 1)


@pytest.mark.parametrize("m,k", [(16450, 40), (8300, 100), (4200, 200), (2100, 401), (1100, 1000), (600, 2000), (270, 3001), (260, 12000), (300, 16500)])
def test_backward_of_more_rows_than_are_taken_at_once(m, k):
    d = inputs(m, k, False, 300 * m + k)
    check_backward(d, (1, 1), False, acc=np.linspace(-3, 3, k).astype(np.float32).astype(np.float64))


def test_backward_parts_of_it():
    for m, k in ((5, 100), (300, 1032), (2, 17000)):
        d = inputs(m, k, False, 12)
        check_backward(d, (1, 1), False, without=VECTORS)
        check_backward(d, (2, 1), False, which=())
        for name in GRADS:
            check_backward(d, (1, 2), False, which=(name,))
        check_backward(d, (1, 1), False, scale=-1.5, ds=False)


def test_no_rows():
    """Sums over no rows are zero, or what was there."""
    for k in (50, 17000):
        d = {n: v[:0] if v.ndim == 2 else v for n, v in inputs(3, k, False, 13).items()}
        assert not any(g.any() for g in backward(d, (1, 1), False)[1][2:])
        start = np.arange(float(k))
        assert all(np.array_equal(g, start) for g in backward(d, (1, 1), False, acc=start)[1][2:])


@pytest.mark.parametrize("kinds", KINDS)
def test_backward_against_differences(kinds):
    """The gradient of sum(y dy + s ds) along a direction, from central differences of the 64-bit forward pass."""
    m, k = 7, 96
    d = inputs(m, k, True, 14)
    rng = np.random.default_rng(15)
    names = ("x", "b") + VECTORS
    v = {n: rng.standard_normal(d[n].shape) for n in names}
    _, got = backward(d, kinds, True)

    def loss(t):
        e = {n: d[n] + t * v[n] for n in names}
        s, *_ = orr.resnorm_s(e["b"], e["x"], SCALE, kinds[0], e["gamma_a"], e["beta_a"], e["gate"], EPS)
        return (orr.resnorm_y(s, kinds[1], e["gamma_b"], e["beta_b"], EPS)[0] * d["dy"]).sum() + (s * d["ds"]).sum()

    slope = (loss(1e-5) - loss(-1e-5)) / 2e-5
    parts = [g * v[n] for g, n in zip(got, names)]
    parts[1] = got[1] * v["b"]  # dB is rounded to bf16: half a step of each value
    assert abs(sum(p.sum() for p in parts) - slope) <= 1e-5 * sum(np.abs(p).sum() for p in parts) + bu.BF16 * np.abs(parts[1]).sum()


def test_offsets_past_32_bits():
    """Rows a billion elements apart."""
    m, k, ld = 3, 1000, (1 << 30) + 8
    d = inputs(m, k, False, 17)
    p = bu.problem(m, k, 0)
    far = [torch.empty(2 * ld + 1024, dtype=torch.bfloat16, device=bu.DEV) for _ in range(2)]
    rows = [t.as_strided((m, k), (ld, 1)) for t in far]
    rows[0].copy_(torch.from_numpy(d["b"]).bfloat16())
    X, Y = bu.Mat(d["x"]), bu.Out(m, k)
    dev, _ = vectors(d)
    st = torch.empty((m, 4), device=bu.DEV)
    axo.axo_resnorm_fwd(p, far[0].data_ptr(), ld, X.ptr, X.ld, 0, 1, bu.ptr(dev["gamma_a"]), bu.ptr(dev["beta_a"]), bu.ptr(dev["gate"]), SCALE, 1, bu.ptr(dev["gamma_b"]),
                        bu.ptr(dev["beta_b"]), EPS, far[1].data_ptr(), ld, Y.ptr, Y.ld, st.data_ptr(), bu.stream())
    S, Yw, stw = forward(d, (1, 1), False)
    assert np.array_equal(rows[1].double().cpu().numpy(), S) and np.array_equal(Y.result(), Yw) and np.array_equal(st.double().cpu().numpy(), stw)


@pytest.mark.parametrize("k", [1000, 17000])
def test_backward_offsets_past_32_bits(k):
    """Rows of all matrices a billion elements apart."""
    m, ld = 3, (1 << 30) + 8
    d = inputs(m, k, False, 19)
    p = bu.problem(m, k, 0)
    (S, stats), want = backward(d, (1, 1), False)
    far = [torch.empty(2 * ld + 17408, dtype=torch.bfloat16, device=bu.DEV) for _ in range(6)]
    rows = [t.as_strided((m, k), (ld, 1)) for t in far]
    for r, v in zip(rows, (d["dy"], d["ds"], d["b"], S)):
        r.copy_(torch.from_numpy(v).bfloat16())
    dev, _ = vectors(d)
    out = [torch.zeros(k, device=bu.DEV) for _ in GRADS]
    ws = torch.empty(axo.axo_resnorm_workspace_bytes(p), dtype=torch.uint8, device=bu.DEV)
    stats = torch.from_numpy(stats).float().to(bu.DEV)
    at = [t.data_ptr() for t in far]
    axo.axo_resnorm_bwd(p, at[0], ld, at[1], ld, at[2], ld, at[3], ld, 0, 1, bu.ptr(dev["gamma_a"]), bu.ptr(dev["beta_a"]), bu.ptr(dev["gate"]), SCALE, 1, bu.ptr(dev["gamma_b"]),
                        stats.data_ptr(), at[4], ld, at[5], ld, *[t.data_ptr() for t in out], 0, ws.data_ptr(), ws.numel(), bu.stream())
    got = [rows[4], rows[5]] + out
    assert all(np.array_equal(a.double().cpu().numpy(), b) for a, b in zip(got, want))


@pytest.mark.parametrize("m,k", [(1, 4096), (37, 1027), (700, 512), (64, 12288), (3, 17000)])
def test_same_bits_on_any_stream_and_in_graphs(m, k):
    d = inputs(m, k, False, 18)
    side = torch.cuda.Stream()
    first = forward(d, (2, 1), False) + tuple(backward(d, (2, 1), False)[1])
    with torch.cuda.stream(side):
        again = forward(d, (2, 1), False) + tuple(backward(d, (2, 1), False)[1])
    assert all(np.array_equal(a, b) for a, b in zip(first, again))

    p = bu.problem(m, k, 0)
    B, X, dY, dS = bu.Mat(d["b"]), bu.Mat(d["x"]), bu.Mat(d["dy"]), bu.Mat(d["ds"])
    S, Y, dX, dB = (bu.Out(m, k) for _ in range(4))
    dev, _ = vectors(d)
    st = torch.zeros((m, 4), device=bu.DEV)
    out = [torch.zeros(k, device=bu.DEV) for _ in GRADS]
    ws = torch.empty(axo.axo_resnorm_workspace_bytes(p), dtype=torch.uint8, device=bu.DEV)

    def both():
        axo.axo_resnorm_fwd(p, B.ptr, B.ld, X.ptr, X.ld, 0, 1, bu.ptr(dev["gamma_a"]), bu.ptr(dev["beta_a"]), bu.ptr(dev["gate"]), SCALE, 1, bu.ptr(dev["gamma_b"]),
                            bu.ptr(dev["beta_b"]), EPS, S.ptr, S.ld, Y.ptr, Y.ld, st.data_ptr(), bu.stream())
        axo.axo_resnorm_bwd(p, dY.ptr, dY.ld, dS.ptr, dS.ld, B.ptr, B.ld, S.ptr, S.ld, 0, 1, bu.ptr(dev["gamma_a"]), bu.ptr(dev["beta_a"]), bu.ptr(dev["gate"]), SCALE, 1,
                            bu.ptr(dev["gamma_b"]), st.data_ptr(), dX.ptr, dX.ld, dB.ptr, dB.ld, *[t.data_ptr() for t in out], 0, ws.data_ptr(), ws.numel(), bu.stream())

    both()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        both()
    results = [S.view(), Y.view(), dX.view(), dB.view(), st] + out
    for turn in range(3):
        B.view().copy_(torch.from_numpy(np.roll(d["b"], turn, axis=1)).bfloat16())
        both()
        torch.cuda.synchronize()
        eager = [t.clone() for t in results]
        for t in results:
            t.fill_(float("nan"))
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(eager, results)), turn
