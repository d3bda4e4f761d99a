"""The residual addition's operators and the orthogonalised update without a GPU: every refusal ahead of the first HIP call, calls with nothing to do, the binding against
the headers, and the 64-bit definitions that the GPU tests compare with."""
import inspect
import math
import os
import re

import numpy as np
import pytest

import paper_2305_13525_amd as axo
from oracle import residual as orr
from paper_2305_13525_amd import residual

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
BAD_GRID, BAD_COORD, INDIVISIBLE, NULL_PTR, MISALIGNED, BAD_LD, WORKSPACE, BAD_EPILOGUE, HIP, BAD_SIZE, BAD_ARG = (-1, -2, -3, -4, -5, -6, -7, -8, -9, -10, -11)


def P(T=64, K=32, N=48, grid=(1, 1, 1), coord=(0, 0, 0), transposed=0):
    return axo.Problem.make(grid, coord, T, K, N, transposed)


def at(n):
    return n << 40  # far from each other, aligned, never dereferenced


GOOD = {
    "axo_fc_add": dict(p=P(), X=at(1), ldx=32, W=at(2), ldw=48, bias=at(3), epilogue=2, R=at(4), ldr=48, type=0, scale=0.5, Z=at(5), ldz=48, Y=at(6), ldy=48, ws=at(9),
                       ws_bytes=1 << 40),
    "axo_fc_add_dact": dict(p=P(), dY=at(1), lddy=48, type=0, Z=at(2), ldz=48, epilogue=3, scale=0.5, dZ=at(3), lddz=48),
    "axo_resnorm_fwd": dict(p=P(), B=at(1), ldb=32, X=at(2), ldx=32, type=0, norm_a=1, gamma_a=at(3), beta_a=at(4), gate=at(5), scale=0.5, norm_b=1, gamma_b=at(6),
                            beta_b=at(7), eps=1e-5, S=at(8), lds=32, Y=at(9), ldy=32, stats=at(10)),
    "axo_resnorm_bwd": dict(p=P(), dY=at(1), lddy=32, dS=at(2), ldds=32, B=at(3), ldb=32, S=at(4), lds=32, type=0, norm_a=1, gamma_a=at(5), beta_a=at(6), gate=at(7),
                            scale=0.5, norm_b=2, gamma_b=at(8), stats=at(9), dX=at(10), lddx=32, dB=at(11), lddb=32, dgamma_a=at(12), dbeta_a=at(13), dgate=at(14),
                            dgamma_b=at(15), dbeta_b=at(16), accumulate=0, ws=at(17), ws_bytes=1 << 30),
    "axo_ortho": dict(p=P(), G=at(1), ldg=48, type=0, steps=5, abc=None, eps=1e-7, O=at(2), ldo=48, ws=at(3), ws_bytes=1 << 40),
}
NAMES = sorted(GOOD)
MATRICES = {"X": "ldx", "W": "ldw", "R": "ldr", "Z": "ldz", "Y": "ldy", "dY": "lddy", "dZ": "lddz", "B": "ldb", "S": "lds", "dS": "ldds", "dX": "lddx", "dB": "lddb", "G": "ldg",
            "O": "ldo"}
OPTIONAL = {("axo_fc_add", "Z"), ("axo_resnorm_bwd", "dS")}
OUTPUTS = {"axo_fc_add": ("Z", "Y"), "axo_fc_add_dact": ("dZ",), "axo_resnorm_fwd": ("S", "Y", "stats"),
           "axo_resnorm_bwd": ("dX", "dB", "dgamma_a", "dbeta_a", "dgate", "dgamma_b", "dbeta_b"), "axo_ortho": ("O",)}
VECTORS = {"bias": 8, "gamma_a": 8, "beta_a": 8, "gate": 8, "gamma_b": 8, "beta_b": 8, "stats": 8, "dgamma_a": 2, "dbeta_a": 2, "dgate": 2, "dgamma_b": 2, "dbeta_b": 2}


def call(name, **changed):
    return getattr(axo, name)(**{**GOOD[name], **changed}, check=False)


@pytest.mark.parametrize("name", NAMES)
def test_problems(name):
    assert call(name, p=P(grid=(0, 1, 1))) == BAD_GRID
    assert call(name, p=P(coord=(1, 0, 0))) == BAD_COORD
    assert call(name, p=P(T=65, grid=(1, 1, 2))) == INDIVISIBLE
    assert call(name, p=P(T=-1)) == BAD_SIZE
    assert call(name, p=P(T=1 << 32)) == BAD_SIZE
    assert call(name, p=P(transposed=2)) == BAD_ARG
    assert call(name, p=None) == NULL_PTR
    p = P()
    p.reserved = 1
    assert call(name, p=p) == BAD_ARG


@pytest.mark.parametrize("name", NAMES)
def test_matrices(name):
    for pointer, ld in MATRICES.items():
        if pointer not in GOOD[name]:
            continue
        if (name, pointer) not in OPTIONAL:
            assert call(name, **{pointer: None}) == NULL_PTR, pointer
        assert call(name, **{pointer: GOOD[name][pointer] + 8}) == MISALIGNED, pointer
        assert call(name, **{ld: 24}) == BAD_LD, ld
        assert call(name, **{ld: GOOD[name][ld] + 4}) == MISALIGNED, ld


@pytest.mark.parametrize("name", NAMES)
def test_vectors(name):
    for v, off in VECTORS.items():
        if v in GOOD[name]:
            assert call(name, **{v: GOOD[name][v] + off}) == MISALIGNED, v
    if name == "axo_resnorm_bwd":
        assert call(name, stats=None) == NULL_PTR


@pytest.mark.parametrize("name", NAMES)
def test_kinds(name):
    good = GOOD[name]
    assert call(name, type=2) == BAD_ARG and call(name, type=-1) == BAD_ARG
    if "epilogue" in good:
        assert call(name, epilogue=4) == BAD_EPILOGUE and call(name, epilogue=-1) == BAD_EPILOGUE
        assert call(name, epilogue=1) == BAD_ARG and call(name, epilogue=0) == BAD_ARG  # Z without an activation
    if "bias" in good:
        for epilogue in (1, 2, 3):
            assert call(name, epilogue=epilogue, bias=None, Z=None) == BAD_EPILOGUE
    if "norm_a" in good:
        assert call(name, norm_a=3) == BAD_ARG and call(name, norm_a=-1) == BAD_ARG and call(name, norm_b=0) == BAD_ARG and call(name, norm_b=3) == BAD_ARG
    if "accumulate" in good:
        assert call(name, accumulate=2) == BAD_ARG
    if "scale" in good:
        for scale in (math.nan, math.inf, -math.inf):
            assert call(name, scale=scale) == BAD_ARG
    if "eps" in good:
        for eps in (-1e-6, math.nan, math.inf):
            assert call(name, eps=eps) == BAD_ARG
    if "steps" in good:
        assert call(name, steps=0) == BAD_ARG and call(name, steps=axo.AXO_ORTHO_MOST_STEPS + 1) == BAD_ARG
        for i in range(6):
            abc = [1.0] * 6
            for bad in (math.nan, math.inf):
                abc[i] = bad
                assert call(name, steps=2, abc=abc) == BAD_ARG
        for n in (0, 5, 7):
            with pytest.raises(ValueError):
                call(name, steps=2, abc=[1.0] * n)


def test_grids():
    """What needs whole rows, whole sums or whole weights, and what does not."""
    for grid, transposed in (((2, 1, 1), 0), ((1, 2, 1), 1)):
        for name in ("axo_resnorm_fwd", "axo_resnorm_bwd", "axo_fc_add", "axo_fc_add_dact", "axo_ortho"):
            assert call(name, p=P(grid=grid, transposed=transposed)) == BAD_GRID, name
        assert call("axo_fc_add", p=P(T=0, grid=grid, transposed=transposed), epilogue=1, Z=None) == 0
        assert call("axo_fc_add_dact", p=P(T=0, grid=grid, transposed=transposed), epilogue=1, Z=None) == 0
    for grid, transposed in (((1, 2, 1), 0), ((2, 1, 1), 1), ((1, 1, 2), 0)):
        for name in ("axo_resnorm_fwd", "axo_fc_add", "axo_fc_add_dact"):
            assert call(name, p=P(T=0, grid=grid, transposed=transposed)) == 0, name
    assert call("axo_ortho", p=P(grid=(1, 2, 1))) == BAD_GRID and call("axo_ortho", p=P(grid=(1, 1, 2), K=0)) == 0
    # of shards that do not add the residual neither it nor the bias is looked at, but for whether there is one
    p = P(T=64, K=64, grid=(2, 1, 1), coord=(1, 0, 0))
    assert call("axo_fc_add", p=p, epilogue=0, bias=None, R=None, Z=None) in (0, HIP)
    assert call("axo_fc_add", p=p, epilogue=0, bias=None, R=at(6), Z=None) in (0, HIP)


@pytest.mark.parametrize("name", NAMES)
def test_shared_bytes(name):
    """Every output against every other matrix or vector of the call."""
    good = GOOD[name]
    pointers = [n for n in good if isinstance(good[n], int) and good[n] >= at(1) and n != "ws_bytes" and not (n == "ws" and name == "axo_fc_add")]  # needs none here
    for out in OUTPUTS[name]:
        for other in pointers:
            if other != out:
                assert call(name, **{out: good[other]}) == BAD_ARG, (out, other)


def test_column_blocks_of_one_buffer_are_apart():
    assert call("axo_resnorm_fwd", p=P(), S=at(8), lds=64, Y=at(8) + 64, ldy=64, X=at(2), ldx=32) in (0, HIP)
    assert call("axo_resnorm_fwd", S=at(8), lds=64, Y=at(8) + 56 + 8 - 16, ldy=64) == BAD_ARG


def test_workspaces():
    p = P(T=4096, K=1024)
    n = axo.axo_resnorm_workspace_bytes(p)
    lds = {ld: 1024 for ld in ("lddy", "ldds", "ldb", "lds", "lddx", "lddb")}
    assert n > 0 and axo.axo_resnorm_workspace_bytes(P(T=4096, K=20000)) > axo.axo_resnorm_workspace_bytes(P(T=4096, K=16384))
    assert call("axo_resnorm_bwd", p=p, ws_bytes=n - 1, **lds) == WORKSPACE and call("axo_resnorm_bwd", p=p, ws=None, **lds) == WORKSPACE
    assert call("axo_resnorm_bwd", p=p, ws=at(17) + 8, **lds) == MISALIGNED and call("axo_resnorm_bwd", p=p, ws=at(11), **lds) == BAD_ARG
    none = {g: None for g in OUTPUTS["axo_resnorm_bwd"][2:]}
    assert call("axo_resnorm_bwd", p=p, ws=None, ws_bytes=0, **lds, **none) in (0, HIP)
    found = 0
    for T, K, N in ((1, 8192, 16384), (1, 16384, 1024), (1, 64, 64), (24, 4096, 512), (4096, 4096, 4096), (0, 4096, 512)):
        p = P(T=T, K=K, N=N)
        n = axo.axo_fc_add_workspace_bytes(p)
        lds = {ld: 16384 for ld in ("ldx", "ldw", "ldr", "ldz", "ldy")}
        if n:
            found += 1
            assert call("axo_fc_add", p=p, ws_bytes=n - 1, **lds) == WORKSPACE and call("axo_fc_add", p=p, ws=None, **lds) == WORKSPACE
            assert call("axo_fc_add", p=p, ws=at(9) + 8, **lds) == MISALIGNED and call("axo_fc_add", p=p, ws=at(6), **lds) == BAD_ARG
    assert found
    n = axo.axo_ortho_workspace_bytes(P())
    assert n > 0 and call("axo_ortho", ws_bytes=n - 1) == WORKSPACE and call("axo_ortho", ws=None) == WORKSPACE and call("axo_ortho", ws=at(3) + 8) == MISALIGNED
    assert call("axo_ortho", ws=at(1)) == BAD_ARG and call("axo_ortho", ws=at(2)) == BAD_ARG
    for f in (axo.axo_resnorm_workspace_bytes, axo.axo_fc_add_workspace_bytes, axo.axo_ortho_workspace_bytes):
        assert f(P(grid=(0, 1, 1))) == 0 and f(P(coord=(1, 0, 0))) == 0
    assert axo.axo_ortho_workspace_bytes(P(grid=(2, 1, 1))) == 0


def test_weights_too_large_to_orthogonalise():
    assert call("axo_ortho", p=P(K=1 << 16, N=1 << 15), ldg=1 << 15, ldo=1 << 15) == BAD_SIZE
    assert axo.axo_ortho_workspace_bytes(P(K=1 << 16, N=1 << 15)) == 0 and axo.axo_ortho_workspace_bytes(P(K=1 << 15, N=65216)) > 0


@pytest.mark.parametrize("name", NAMES)
def test_nothing_to_do(name):
    """No tokens, or no columns: accepted without a launch, pointers and leading dimensions unseen."""
    nothing = {k: None for k, v in GOOD[name].items() if isinstance(v, int) and v >= at(1) and k not in ("ws_bytes", "W", "bias")}
    lds = {k: 0 for k in GOOD[name] if k.startswith("ld") and k != "ldw"}
    if name in ("axo_resnorm_bwd", "axo_ortho"):
        assert call(name, p=P(K=0), **nothing, **lds) == 0
    else:
        if "Z" in nothing and name == "axo_fc_add":
            nothing["epilogue"] = 1
        assert call(name, p=P(T=0), **nothing, **lds) == 0


def test_binding_matches_headers():
    """Names, order and kinds of the arguments of every function of the headers."""
    kinds = {"int64_t": "l", "int": "i", "float": "f", "size_t": "z"}
    found = {}
    for header in ("axo_residual.h", "axo_update.h"):
        text = re.sub(r"/\*.*?\*/", "", open(os.path.join(ROOT, "include", header)).read(), flags=re.S)
        for name, args in re.findall(r"\bint (axo_\w+)\(([^)]*)\);", text):
            found[name] = "".join("p" if "axo_problem_t" in a else "v" if "*" in a else kinds[a.split()[0]] for a in args.split(","))
            names = [re.split(r"[\s*]+", a.strip())[-1] for a in args.split(",")]
            assert list(inspect.signature(getattr(axo, name)).parameters) == [("stream" if n == "hip_stream" else n) for n in names] + ["check"], name
    assert sorted(found) == NAMES and found.pop("axo_ortho") == "pvliivfvlvzv"
    assert found == residual._SIGNATURES


def test_errors_are_raised():
    for name, bad in (("axo_fc_add", dict(epilogue=9)), ("axo_resnorm_bwd", dict(type=9)), ("axo_ortho", dict(steps=0))):
        with pytest.raises(axo.AxoError, match=name):
            getattr(axo, name)(**{**GOOD[name], **bad})


def outcome(f, *a, **k):
    try:
        return f(*a, **k)
    except Exception as e:  # noqa: BLE001
        return type(e), str(e)


@pytest.mark.parametrize("name", sorted(residual._SIGNATURES))
def test_quick_calls(name):
    """The extension module's calls against the ctypes wrappers: the same status or exception for every form of arguments, none of which launches anything."""
    _calls = pytest.importorskip("paper_2305_13525_amd._calls", reason="the extension module is not built")
    quick, wrapper = getattr(_calls, name), residual._WRAPPERS[name]
    assert getattr(axo, name) is quick and quick is not wrapper
    axo.axo_fc_add_workspace_bytes(P())  # the library is loaded
    plain = [None if isinstance(v, int) and v >= at(1) and k != "ws_bytes" else v for k, v in GOOD[name].items()]
    if name == "axo_fc_add":
        plain[6] = 0
    empty = [P(T=0, K=0, N=0)] + plain[1:]
    assert outcome(quick, *empty) == outcome(wrapper, *empty) == 0
    n = 0
    for base in (empty, [P(grid=(0, 1, 1))] + plain[1:]):
        for i in range(len(base)):
            for v in (None, 1.5, "x", True, -1, 2 ** 31, 2 ** 63, 2 ** 64, 7):
                if i == 0 and isinstance(v, int):
                    continue
                args = base[:i] + [v] + base[i + 1:]
                assert outcome(quick, *args, check=False) == outcome(wrapper, *args, check=False), args
                assert outcome(quick, *args, None, False) == outcome(wrapper, *args, None, False), args
                n += 1
        for m in range(len(base)):
            assert outcome(quick, *base[:m]) == outcome(wrapper, *base[:m])
    assert n > 100


# ---- the definitions ----

def test_definition_of_the_norms():
    b = np.array([[1.0, 2.0, 3.0, 6.0]])
    s, mean, rstd = orr.resnorm_s(b, np.full((1, 4), 10.0), 2.0, orr.LAYER, np.array([1.0, 1.0, 2.0, 1.0]), np.array([0.0, 0.0, 0.0, 10.0]), np.array([1.0, 2.0, 1.0, 0.5]), 0.5)
    assert mean[0] == 3.0 and rstd[0] == 0.5  # deviations -2 -1 0 3, squares 14 / 4 = 3.5
    assert np.array_equal(s, [[8.0, 8.0, 10.0, 21.5]])
    s, mean, rstd = orr.resnorm_s(b, np.zeros((1, 4)), 1.0, orr.RMS, eps=3.5)
    assert mean[0] == 0.0 and rstd[0] == 0.25 and np.array_equal(s, b / 4)  # squares 50 / 4 = 12.5
    assert np.array_equal(orr.resnorm_s(b, b, 0.5, orr.NONE)[0], 1.5 * b)


@pytest.mark.parametrize("kinds", [(a, b) for a in range(3) for b in (1, 2)])
def test_gradients_of_the_definitions(kinds):
    rng = np.random.default_rng(0)
    m, k = 5, 9
    d = {n: rng.standard_normal((m, k)) for n in ("x", "b", "dy", "ds")}
    for n in ("gamma_a", "beta_a", "gate", "gamma_b", "beta_b"):
        d[n] = rng.standard_normal(k)

    def forward(e):
        s, *first = orr.resnorm_s(e["b"], e["x"], 0.7, kinds[0], e["gamma_a"], e["beta_a"], e["gate"])
        y, *second = orr.resnorm_y(s, kinds[1], e["gamma_b"], e["beta_b"])
        return s, y, np.stack(first + second, 1)

    s, _, stats = forward(d)
    grads = orr.resnorm_bwd(d["dy"], d["ds"], d["b"], s, stats, 0.7, *kinds, d["gamma_a"], d["beta_a"], d["gate"], d["gamma_b"])
    for name, grad in zip(("x", "b", "gamma_a", "beta_a", "gate", "gamma_b", "beta_b"), grads):
        v = rng.standard_normal(d[name].shape)

        def loss(t):
            s, y, _ = forward({**d, name: d[name] + t * v})  # noqa: B023
            return (s * d["ds"]).sum() + (y * d["dy"]).sum()

        assert abs((loss(1e-5) - loss(-1e-5)) / 2e-5 - (grad * v).sum()) < 1e-7, name


def test_definition_of_the_update():
    """On singular values, whichever side is longer; zeros stay."""
    rng = np.random.default_rng(1)
    u, _, v = np.linalg.svd(rng.standard_normal((12, 7)), full_matrices=False)
    sv = np.linspace(0.1, 1.0, 7)
    sv /= np.linalg.norm(sv)
    want = sv.copy()
    for _ in range(3):
        want = orr.QUINTIC[0] * want + orr.QUINTIC[1] * want ** 3 + orr.QUINTIC[2] * want ** 5
    g = (u * sv) @ v * 42.0
    assert np.allclose(orr.ortho(g, 3), (u * want) @ v, atol=1e-12) and np.allclose(orr.ortho(g.T, 3), ((u * want) @ v).T, atol=1e-12)
    assert not orr.ortho(np.zeros((3, 4)), 2).any()
    path = []
    orr.ortho(g, 3, path=path)
    assert len(path) == 3 and path[0].shape == (7, 12)
