"""Layer norm and the gated block without a GPU: every refusal ahead of the first HIP call, calls with nothing to do, the binding against the
header, and the 64-bit definitions that the GPU tests compare with."""
import inspect
import math
import os
import re

import numpy as np
import pytest

import paper_2305_13525_amd as axo
from oracle import block as ob
from paper_2305_13525_amd import block

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
BAD_GRID, BAD_COORD, INDIVISIBLE, NULL_PTR, MISALIGNED, BAD_LD, WORKSPACE, BAD_EPILOGUE, HIP, BAD_SIZE, BAD_ARG = (-1, -2, -3, -4, -5, -6, -7, -8, -9, -10, -11)


def P(T=64, K=32, N=48, grid=(1, 1, 1), coord=(0, 0, 0), transposed=0):
    return axo.Problem.make(grid, coord, T, K, N, transposed)


def at(n):
    return n << 40  # far from each other, aligned, never dereferenced


# plain arguments of each entry point; all of them are accepted but for the launch, which has no device here
GOOD = {
    "axo_norm_fwd": dict(p=P(), X=at(1), ldx=32, R=at(2), ldr=32, type=0, gamma=at(3), beta=at(4), eps=1e-5, S=at(5), lds=32, Y=at(6), ldy=32, stats=at(7)),
    "axo_norm_part": dict(p=P(), X=at(1), ldx=32, R=at(2), ldr=32, type=0, S=at(5), lds=32, part=at(7)),
    "axo_norm_apply": dict(p=P(), S=at(1), lds=32, type=0, parts=at(2), n_parts=1, gamma=at(3), beta=at(4), eps=1e-5, Y=at(6), ldy=32, stats=at(7)),
    "axo_norm_bwd": dict(p=P(), dY=at(1), lddy=32, S=at(2), lds=32, R=at(3), ldr=32, type=0, gamma=at(4), stats=at(5), dX=at(6), lddx=32, dgamma=at(7),
                         dbeta=at(8), accumulate=0, ws=at(9), ws_bytes=1 << 30),
    "axo_norm_bwd_part": dict(p=P(), dY=at(1), lddy=32, S=at(2), lds=32, type=0, gamma=at(4), stats=at(5), sums=at(6), dgamma=at(7), dbeta=at(8),
                              accumulate=0, ws=at(9), ws_bytes=1 << 30),
    "axo_norm_bwd_apply": dict(p=P(), dY=at(1), lddy=32, S=at(2), lds=32, R=at(3), ldr=32, type=0, gamma=at(4), stats=at(5), sums=at(6), dX=at(7), lddx=32),
    "axo_gated_fwd": dict(p=P(), X=at(1), ldx=32, Wg=at(2), Wu=at(3), ldw=48, bg=at(4), bu=at(5), gate=0, G=at(6), U=at(7), ldz=48, H=at(8), ldh=48,
                          ws=at(9), ws_bytes=1 << 40),
    "axo_gated_act": dict(p=P(), G=at(1), U=at(2), ldz=32, gate=0, H=at(3), ldh=32),
    "axo_gated_dact": dict(p=P(), dH=at(1), lddh=32, G=at(2), U=at(3), ldz=32, gate=0, dG=at(4), dU=at(5), lddz=32),
    "axo_gated_dgrad_act": dict(p=P(), dY=at(1), lddy=48, W=at(2), ldw=48, G=at(3), U=at(4), ldz=32, gate=0, dG=at(5), dU=at(6), lddz=32, ws=at(9), ws_bytes=1 << 40),
    "axo_gated_dgrad": dict(p=P(), dG=at(1), dU=at(2), lddz=48, Wg=at(3), Wu=at(4), ldw=48, dX=at(5), lddx=32, ws=at(9), ws_bytes=1 << 40),
    "axo_gated_wgrad": dict(p=P(), X=at(1), ldx=32, dG=at(2), dU=at(3), lddz=48, dWg=at(4), dWu=at(5), lddw=48, ws=at(9), ws_bytes=1 << 40),
    "axo_gated_wgrad_acc": dict(p=P(), X=at(1), ldx=32, dG=at(2), dU=at(3), lddz=48, dWg=at(4), dWu=at(5), lddw=48, ws=at(9), ws_bytes=1 << 40),
}
NAMES = sorted(GOOD)
OPTIONAL = {"R", "gamma", "beta", "stats", "dgamma", "dbeta", "bg", "bu", "ws", "stream"}
REQUIRED_STATS = {"axo_norm_bwd", "axo_norm_bwd_part", "axo_norm_bwd_apply"}


def call(name, **changed):
    return getattr(axo, name)(**{**GOOD[name], **changed}, check=False)


def matrices(name):
    """(pointer, leading dimension) names of the call's matrices."""
    pairs = []
    for pointer, ld in (("X", "ldx"), ("R", "ldr"), ("S", "lds"), ("Y", "ldy"), ("dY", "lddy"), ("dX", "lddx"), ("Wg", "ldw"), ("Wu", "ldw"), ("W", "ldw"),
                        ("G", "ldz"), ("U", "ldz"), ("H", "ldh"), ("dH", "lddh"), ("dG", "lddz"), ("dU", "lddz"), ("dWg", "lddw"), ("dWu", "lddw")):
        if pointer in GOOD[name]:
            pairs.append((pointer, ld))
    return pairs


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
    for pointer, ld in matrices(name):
        if pointer != "R":  # without it S is not looked at
            assert call(name, **{pointer: None}) == NULL_PTR, pointer
        assert call(name, **{pointer: GOOD[name][pointer] + 8}) == MISALIGNED, pointer
        assert call(name, **{ld: 24}) == BAD_LD, ld
        assert call(name, **{ld: GOOD[name][ld] + (2 if name.endswith("_acc") and ld == "lddw" else 4)}) == MISALIGNED, ld


@pytest.mark.parametrize("name", NAMES)
def test_vectors(name):
    for v, off in (("gamma", 8), ("beta", 8), ("bg", 8), ("bu", 8), ("stats", 4), ("part", 4), ("parts", 4), ("sums", 4), ("dgamma", 2), ("dbeta", 2)):
        if v not in GOOD[name]:
            continue
        assert call(name, **{v: GOOD[name][v] + off}) == MISALIGNED, v
        if v not in OPTIONAL or (v == "stats" and name in REQUIRED_STATS):
            assert call(name, **{v: None}) == NULL_PTR, v


@pytest.mark.parametrize("name", NAMES)
def test_kinds(name):
    good = GOOD[name]
    if "type" in good:
        assert call(name, type=2) == BAD_ARG and call(name, type=-1) == BAD_ARG
    if "gate" in good:
        assert call(name, gate=3) == BAD_EPILOGUE and call(name, gate=-1) == BAD_EPILOGUE
    if "accumulate" in good:
        assert call(name, accumulate=2) == BAD_ARG
    if "eps" in good:
        for eps in (-1e-6, math.nan, math.inf):
            assert call(name, eps=eps) == BAD_ARG
    if "n_parts" in good:
        assert call(name, n_parts=2) == BAD_ARG and call(name, n_parts=0) == BAD_ARG
        assert call(name, p=P(grid=(2, 1, 1))) == BAD_ARG and call(name, p=P(grid=(1, 2, 1), transposed=1)) == BAD_ARG


@pytest.mark.parametrize("name", NAMES)
def test_shared_bytes(name):
    """Every output against every other matrix or vector of the call, and no two inputs."""
    good = GOOD[name]
    outputs = [n for n in ("S", "Y", "stats", "part", "sums", "dX", "dgamma", "dbeta", "H", "dG", "dU", "dWg", "dWu", "G", "U") if n in good]
    if not name.startswith("axo_norm_fwd") and name != "axo_norm_part" and "S" in outputs:
        outputs.remove("S")
    if name != "axo_norm_fwd" and name != "axo_norm_apply" and "stats" in outputs:
        outputs.remove("stats")
    if name == "axo_norm_bwd_apply":
        outputs.remove("sums")
    if name != "axo_gated_fwd":
        outputs = [n for n in outputs if n not in ("G", "U")]
    if name in ("axo_gated_dgrad", "axo_gated_wgrad", "axo_gated_wgrad_acc"):
        outputs = [n for n in outputs if n not in ("dG", "dU")]
    pointers = [n for n in good if isinstance(good[n], int) and good[n] >= at(1)]
    assert outputs
    for out in outputs:
        for other in pointers:
            if other != out and other != "ws":
                assert call(name, **{out: good[other]}) == BAD_ARG, (out, other)


def test_column_blocks_of_one_buffer_are_apart():
    wide = dict(ldz=96, G=at(6), U=at(6) + 96)
    p = P(T=0)
    assert call("axo_gated_fwd", p=p, **wide) == 0
    # found apart although their ranges interleave: the call gets as far as the launch, or there is no device error to tell
    assert call("axo_gated_wgrad", dWg=at(4), dWu=at(4) + 96, lddw=96) in (0, HIP)
    assert call("axo_gated_wgrad", dWg=at(4), dWu=at(4) + 80, lddw=96) == BAD_ARG
    assert call("axo_gated_wgrad", dWg=at(4), dWu=at(4) + 96, lddw=88) == BAD_ARG


def test_split_width():
    for grid, transposed in (((2, 1, 1), 0), ((1, 2, 1), 1)):
        assert call("axo_norm_fwd", p=P(grid=grid, transposed=transposed)) == BAD_GRID
        assert call("axo_norm_bwd", p=P(grid=grid, transposed=transposed)) == BAD_GRID
    for grid, transposed in (((1, 2, 1), 0), ((2, 1, 1), 1), ((1, 1, 2), 0)):
        assert call("axo_norm_fwd", p=P(T=0, grid=grid, transposed=transposed)) == 0


def test_workspaces():
    p = P(T=4096, K=1024)
    n = axo.axo_norm_workspace_bytes(p)
    assert n > 0
    for name in ("axo_norm_bwd", "axo_norm_bwd_part"):
        lds = {k: 1024 for k in ("lddy", "lds", "ldr", "lddx") if k in GOOD[name]}
        assert call(name, p=p, ws_bytes=n - 1, **lds) == WORKSPACE and call(name, p=p, ws=None, **lds) == WORKSPACE
        assert call(name, p=p, ws=at(9) + 8, **lds) == MISALIGNED
        assert call(name, p=p, ws=GOOD[name]["dgamma"], **lds) == BAD_ARG
    # a single token through the longest and the shortest reductions, and no tokens
    for T, K, N in ((1, 8192, 16384), (1, 64, 64), (24, 4096, 512), (4096, 4096, 4096), (0, 4096, 512)):
        p = P(T=T, K=K, N=N)
        n = axo.axo_gated_workspace_bytes(p)
        if n:
            for name in ("axo_gated_fwd", "axo_gated_dgrad_act", "axo_gated_dgrad", "axo_gated_wgrad", "axo_gated_wgrad_acc"):
                lds = {k: 16384 for k in ("ldx", "ldw", "ldz", "ldh", "lddy", "lddz", "lddx", "lddw") if k in GOOD[name]}
                assert call(name, p=p, ws_bytes=n - 1, **lds) == WORKSPACE and call(name, p=p, ws=None, **lds) == WORKSPACE
                assert call(name, p=p, ws=at(9) + 8, **lds) == MISALIGNED
    assert axo.axo_norm_workspace_bytes(P(grid=(0, 1, 1))) == 0 and axo.axo_gated_workspace_bytes(P(coord=(1, 0, 0))) == 0


@pytest.mark.parametrize("name", NAMES)
def test_nothing_to_do(name):
    """No tokens, or no columns: accepted without a launch, pointers and leading dimensions unseen."""
    nothing = {k: None for k, v in GOOD[name].items() if isinstance(v, int) and v >= at(1) and k != "ws_bytes"}
    lds = {k: 0 for k in GOOD[name] if k.startswith("ld")}
    if name == "axo_gated_wgrad" or name == "axo_gated_wgrad_acc":
        assert call(name, p=P(T=64, K=0), **{**nothing, "dG": at(2), "dU": at(3)}, **{**lds, "lddz": 48}) == 0
        assert call(name, p=P(T=64, N=0), **{**nothing, "X": at(1)}, **{**lds, "ldx": 32}) == 0
    else:  # weights have elements without tokens, too
        weights = {k: GOOD[name][k] for k in ("Wg", "Wu", "W", "ldw") if k in GOOD[name]}
        assert call(name, p=P(T=0, K=32, N=48), **{**nothing, **lds, **weights}) == 0


def test_binding_matches_header():
    """Names, order and kinds of the arguments of every function of the header."""
    text = open(os.path.join(ROOT, "include", "axo_block.h")).read()
    text = re.sub(r"/\*.*?\*/", "", text, flags=re.S)
    kinds = {"int64_t": "l", "int": "i", "float": "f", "size_t": "z"}
    found = {}
    for name, args in re.findall(r"\bint (axo_\w+)\(([^)]*)\);", text):
        found[name] = "".join("p" if "axo_problem_t" in a else "v" if "*" in a else kinds[a.split()[0]] for a in args.split(","))
        if name == "axo_gated_tiles":  # a query: returns its numbers
            continue
        names = [re.split(r"[\s*]+", a.strip())[-1] for a in args.split(",")]
        taken = list(inspect.signature(getattr(axo, name)).parameters)
        assert taken == [("stream" if n == "hip_stream" else n) for n in names] + ["check"], name
    assert found.pop("axo_gated_tiles") == "pivvv"
    assert found == block._SIGNATURES
    assert sorted(found) == NAMES


def test_errors_are_raised():
    with pytest.raises(axo.AxoError, match="axo_gated_fwd"):
        axo.axo_gated_fwd(**{**GOOD["axo_gated_fwd"], "gate": 9})
    with pytest.raises(axo.AxoError, match="axo_norm_fwd"):
        axo.axo_norm_fwd(**{**GOOD["axo_norm_fwd"], "type": 9})


# ---- the definitions ----

def test_definition_of_the_norm():
    y, mean, rstd = ob.norm_fwd(np.array([[1.0, 2.0, 3.0, 6.0]]), np.array([1.0, 1.0, 2.0, 1.0]), np.array([0.0, 0.0, 0.0, 10.0]), eps=0.5)
    assert mean[0] == 3.0 and rstd[0] == 0.5  # deviations -2 -1 0 3, squares 14 / 4 = 3.5
    assert np.array_equal(y, [[-1.0, -0.5, 0.0, 11.5]])


def test_gradients_of_the_definitions():
    rng = np.random.default_rng(0)
    m, k, f = 5, 9, 7
    x, dy, gamma, beta = rng.standard_normal((m, k)), rng.standard_normal((m, k)), rng.standard_normal(k), rng.standard_normal(k)
    _, mean, rstd = ob.norm_fwd(x, gamma, beta)
    grads = ob.norm_bwd(dy, x, mean, rstd, gamma)
    for i, start in enumerate((x, gamma, beta)):
        v = rng.standard_normal(start.shape)
        loss = lambda t: (ob.norm_fwd(*[a + t * v if j == i else a for j, a in enumerate((x, gamma, beta))])[0] * dy).sum()  # noqa: E731, B023
        assert abs((loss(1e-5) - loss(-1e-5)) / 2e-5 - (grads[i] * v).sum()) < 1e-8
    wg, wu = rng.standard_normal((k, f)), rng.standard_normal((k, f))
    dh = rng.standard_normal((m, f))
    for kind in range(3):
        h, g, u = ob.gated_fwd(x, wg, wu, kind)
        dg, du = ob.gated_dact(dh, g, u, kind)
        for i, grad in ((0, ob.gated_dgrad(dg, du, wg, wu)), (1, x.T @ dg), (2, x.T @ du)):
            v = rng.standard_normal(grad.shape)
            loss = lambda t: (ob.gated_fwd(*[a + t * v if j == i else a for j, a in enumerate((x, wg, wu))], kind)[0] * dh).sum()  # noqa: E731, B023
            assert abs((loss(1e-6) - loss(-1e-6)) / 2e-6 - (grad * v).sum()) < 1e-6


def test_activations():
    """Known values: act(0) = 0, act'(0) = 1/2, limits, SiLU(1) = 1 / (1 + 1/e), GELU(1) = Phi(1)."""
    for kind in range(3):
        value, slope = ob.gate(np.array([0.0, 30.0, -30.0]), kind)
        assert value[0] == 0.0 and slope[0] == 0.5 and abs(value[1] - 30.0) < 1e-10 and abs(value[2]) < 1e-10 and abs(slope[1] - 1.0) < 1e-10
    assert abs(ob.gate(np.array([1.0]), 0)[0][0] - 1.0 / (1.0 + math.exp(-1.0))) < 1e-15
    assert abs(ob.gate(np.array([1.0]), 2)[0][0] - 0.8413447460685429) < 1e-15
    assert abs(ob.gate(np.array([1.0]), 1)[0][0] - 0.8411919906082768) < 1e-12


# ---- the extension module's calls against the ctypes wrappers ----

def outcome(f, *a, **k):
    try:
        return f(*a, **k)
    except Exception as e:  # noqa: BLE001
        return type(e), str(e)


@pytest.mark.parametrize("name", NAMES)
def test_quick_calls(name):
    """The same status or exception for every form of arguments, none of which launches anything: two of them are wrong, or there are no elements."""
    _calls = pytest.importorskip("paper_2305_13525_amd._calls", reason="the extension module is not built")
    quick, wrapper = getattr(_calls, name), block._WRAPPERS[name]
    assert getattr(axo, name) is quick and quick is not wrapper
    axo.axo_gated_workspace_bytes(P())  # the library is loaded
    plain = [None if isinstance(v, int) and v >= at(1) and k != "ws_bytes" else v for k, v in GOOD[name].items()]
    empty = [P(T=0)] + plain[1:] if "wgrad" not in name else [P(T=0, K=0, N=0)] + plain[1:]
    if "Wg" in GOOD[name] or "W" in GOOD[name]:
        empty[0] = P(T=0, K=0, N=0)
    assert outcome(quick, *empty) == outcome(wrapper, *empty) == 0
    n = 0
    for base in (empty, [P(grid=(0, 1, 1))] + plain[1:]):
        for i in range(len(base)):
            for v in (None, 1.5, "x", True, -1, 2 ** 31, 2 ** 63, 2 ** 64, 7):
                args = list(base)
                args[i] = v
                if i == 0 and isinstance(v, int):
                    continue
                for tail in ((), (None, False) if len(base) == len(GOOD[name]) else ()):
                    assert outcome(quick, *args, *tail, check=False) == outcome(wrapper, *args, *tail, check=False) if not tail else outcome(
                        quick, *args, *tail) == outcome(wrapper, *args, *tail), (args, tail)
                    n += 1
        for m in range(len(base)):
            assert outcome(quick, *base[:m]) == outcome(wrapper, *base[:m])
    assert n > 100


# tokens x width x inner width whose outputs have more 64 x 64 tiles than a launch takes, but not more 256-row ones: the large tiles, as axo_fc_fwd
@pytest.mark.parametrize("T,K,N", [(4200000, 64, 4096), (8388608, 64, 2048), (33554432, 64, 512)])
def test_tall_outputs_run_on_tiles(T, K, N):
    assert axo.axo_gated_tiles(P(T, K, N), axo.AXO_GATED_OP_FWD)[1] == (256, 128, 1)
    assert axo.axo_gated_tiles(P(T, 2 * N, K), axo.AXO_GATED_OP_DGRAD_ACT)[1] == (256, 256, 1)
    assert axo.axo_gated_tiles(P(T, 2 * N, K), axo.AXO_GATED_OP_DGRAD)[1] == (256, 256, 1)


def test_what_no_launch_takes_goes_to_the_general_kernel():
    """A billion rows of one column: no tiles, and more rows than the general kernel has a grid for."""
    p = P(2 ** 31 - 1, 8, 8)
    assert axo.axo_gated_tiles(p, axo.AXO_GATED_OP_FWD)[1] == (0, 0, 0)
    assert call("axo_gated_fwd", p=p, **{k: 8 for k in ("ldx", "ldw", "ldz", "ldh")}) == BAD_SIZE
