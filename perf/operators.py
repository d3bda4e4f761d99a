"""Layer norm and the gated feed-forward block, forward and backward, as timed cases: one GPU's share of the sublayer
x + down( act(n Wg) * (n Wu) ), n = norm(x), on buffers that the program owns.

A case gives tokens T, width K and, for the gated block, its inner width F, and which operator is called:

  how = "norm_fwd"    Y = norm(S), S = X (+ residual), with the rows' (mean, 1 / deviation) kept for the backward pass
  how = "norm_bwd"    dX (+ the residual's gradient), dgamma, dbeta
  how = "gated_fwd"   H = act(X Wg + bg) * (X Wu + bu); with `save` also G and U, which the backward pass reads
  how = "gated_dact"  dH = dY Wd^T of the layer below the block's output (K columns), taken through the activation:
                      dG = dH U act'(G), dU = dH act(G); with K = 0 dH is what the program has in hand
  how = "gated_back"  dX = dG Wg^T + dU Wu^T, dWg = X^T dG, dWu = X^T dU

  act   gate's activation: 0 SiLU, 1 GELU (tanh form), 2 GELU (erf form)
  res   the residual is added on the way in (norm_fwd: S is written, too), its gradient on the way out (norm_bwd)
  wide  the residual stream (X, residual, S, dX) in fp32, else bf16
  bias  the two projections have biases
  gap   elements between the end of a matrix row (rounded up to 8) and the next row

Inputs: activations N(0, 1) (the residual stream with a mean and a larger deviation), weights and biases N(0, 0.02),
gammas around 1; bf16 unless said otherwise, accumulators fp32.
"""
import functools
import math

import torch

own = False

DEV = "cuda:0"
SIGMA_W = 0.02
EPS = 1e-5


def _case(name, how, T, K, F=0, act=0, res=False, wide=False, bias=False, save=False, gap=0):
    return {"name": name, "how": how, "T": T, "K": K, "F": F, "act": act, "res": res, "wide": wide, "bias": bias, "save": save, "gap": gap}


def listed():
    return [
        # one token of an answer on its way into a 4096-wide layer, added to the residual stream: nothing but latency
        _case("norm_fwd_token", "norm_fwd", 1, 4096, res=True),
        # the norm ahead of a 12288-wide model's MLP, the tokens of one of four token shards
        _case("norm_fwd_12288", "norm_fwd", 4096, 12288, res=True),
        # nothing is a multiple of anything, an fp32 residual stream with padded rows
        _case("norm_bwd_odd", "norm_bwd", 1001, 1027, wide=True, gap=8),
        # the norm of a 7168-wide (20B) model's block in training, the residual's gradient added
        _case("norm_bwd_7168", "norm_bwd", 8192, 7168, res=True),
        # one token through an 8192-wide model's gated block, inner width 32768 over two GPUs: the weights are what is read
        _case("gated_fwd_token", "gated_fwd", 1, 8192, 16384),
        # a batch of answers, one token each
        _case("gated_fwd_few", "gated_fwd", 24, 4096, 12288, act=1, bias=True),
        # a ragged prompt on a small layer
        _case("gated_fwd_odd", "gated_fwd", 1001, 1027, 515, act=2, bias=True, save=True, gap=8),
        # a training step's tokens through the 8192-wide model's block, what the backward pass reads is kept
        _case("gated_fwd_8192", "gated_fwd", 4096, 8192, 16384, save=True),
        # back through the activation of a ragged mid-size block
        _case("gated_dact_ragged", "gated_dact", 4000, 2000, 6000, act=1),
        # and of the 8192-wide model's
        _case("gated_dact_8192", "gated_dact", 4096, 8192, 16384),
        # the products of a short batch's backward pass: fewer tokens than a tile has rows
        _case("gated_back_few", "gated_back", 96, 2048, 6144),
        # and of a 7168-wide model's training step: the largest
        _case("gated_back_7168", "gated_back", 4096, 7168, 14336),
    ]


def _log_size(rng, lo, hi):
    """A size spread over the logarithm of [lo, hi]: a third of them any number, a third multiples of 8, the rest multiples of 128."""
    v = math.exp(rng.uniform(math.log(lo), math.log(hi)))
    unit = rng.choice((1, 8, 128))
    return min(hi, max(1, lo if v < lo else int(v / unit + 0.5) * unit or unit))


def draw(rng):
    how = rng.choice(("norm_fwd", "norm_bwd", "gated_fwd", "gated_fwd", "gated_dact", "gated_back"))
    gap = rng.choice((0, 0, 0, 8, 64))
    while True:
        t, k, f = _log_size(rng, 1, 16384), _log_size(rng, 32, 16384), _log_size(rng, 32, 16384)
        if how.startswith("norm"):
            if t * k <= 1 << 26:
                f = 0
                break
        elif 1.0 * t * k * f <= 1e11:
            break
    if how == "gated_dact" and rng.random() < 0.3:
        k = 0
    c = _case("", how, t, k, f, gap=gap)
    del c["name"]
    if how.startswith("norm"):
        c["res"], c["wide"] = rng.random() < 0.5, rng.random() < 0.3
    elif how != "gated_back":
        c["act"] = rng.randint(0, 2)
    if how == "gated_fwd":
        c["bias"], c["save"] = rng.random() < 0.4, rng.random() < 0.5
    return c


def _rows(rows, cols, gap, dtype=torch.bfloat16):
    return torch.zeros((rows, (cols + 7) // 8 * 8 + gap), dtype=dtype, device=DEV)[:, :cols]


def _inputs(case, seed):
    """What the operator reads, made on the GPU from the seed alone."""
    how, m, k, f = case["how"], case["T"], case["K"], case["F"]
    gen = torch.Generator(device=DEV)
    gen.manual_seed(seed)

    def normal(rows, cols, sigma=1.0, mean=0.0, dtype=torch.bfloat16, gap=case["gap"]):
        a = torch.empty((rows, (cols + 7) // 8 * 8 + gap), dtype=dtype, device=DEV)
        a.normal_(mean, sigma, generator=gen)
        return a[:, :cols]

    stream = torch.float32 if case["wide"] else torch.bfloat16
    t = {}
    if how.startswith("norm"):
        t["X"] = normal(m, k, 1.5, 0.25, stream)
        if case["res"]:
            t["R"] = normal(m, k, 1.0, 0.0, stream)
        t["gamma"], t["beta"] = normal(1, k, 0.1, 1.0, gap=0)[0], normal(1, k, 0.1, gap=0)[0]
        if how == "norm_bwd":
            t["dY"] = normal(m, k)
            x = t["X"].double()
            mean = x.mean(1)
            rstd = torch.rsqrt((x - mean[:, None]).square().mean(1) + EPS)
            t["stats"] = torch.stack((mean, rstd), 1).float()  # what the forward pass kept
        return t
    if how == "gated_dact":
        if k:
            t["dY"], t["Wd"] = normal(m, k), normal(f, k, SIGMA_W)
        else:
            t["dH"] = normal(m, f)
        t["G"], t["U"] = normal(m, f, 1.5), normal(m, f, 1.5)
        return t
    t["X"], t["Wg"], t["Wu"] = normal(m, k), normal(k, f, SIGMA_W), normal(k, f, SIGMA_W)
    if how == "gated_back":
        t["dG"], t["dU"] = normal(m, f), normal(m, f)
    elif case["bias"]:
        t["bg"], t["bu"] = normal(1, f, SIGMA_W, gap=0)[0], normal(1, f, SIGMA_W, gap=0)[0]
    return t


def prepare(case, seed):
    """The inputs, and the buffers that the program has for the outputs."""
    how, m, k, f, gap = case["how"], case["T"], case["K"], case["F"], case["gap"]
    t = _inputs(case, seed)
    stream = torch.float32 if case["wide"] else torch.bfloat16
    if how == "norm_fwd":
        t["Y"], t["stats"] = _rows(m, k, gap), torch.zeros((m, 2), device=DEV)
        if case["res"]:
            t["S"] = _rows(m, k, gap, stream)
    elif how == "norm_bwd":
        t["dX"] = _rows(m, k, gap, stream)
        t["dgamma"], t["dbeta"] = torch.zeros(k, device=DEV), torch.zeros(k, device=DEV)
    elif how == "gated_fwd":
        t["H"] = _rows(m, f, gap)
        if case["save"]:
            t["Gs"], t["Us"] = _rows(m, f, gap), _rows(m, f, gap)
    elif how == "gated_dact":
        t["dG"], t["dU"] = _rows(m, f, gap), _rows(m, f, gap)
    else:
        t["dX"], t["dWg"], t["dWu"] = _rows(m, k, gap), _rows(k, f, gap), _rows(k, f, gap)
    t["case"], t["stream"] = case, torch.cuda.current_stream().cuda_stream
    return t


def _gate(g, act):
    if act == 0:
        return g / (1.0 + torch.exp(-g))
    if act == 1:
        return 0.5 * g * (1.0 + torch.tanh(math.sqrt(2.0 / math.pi) * (g + 0.044715 * g * g * g)))
    return 0.5 * g * (1.0 + torch.erf(g * math.sqrt(0.5)))


def _dgate(g, act):
    if act == 0:
        s = 1.0 / (1.0 + torch.exp(-g))
        return s * (1.0 + g * (1.0 - s))
    if act == 1:
        th = torch.tanh(math.sqrt(2.0 / math.pi) * (g + 0.044715 * g * g * g))
        return 0.5 * (1.0 + th) + 0.5 * g * (1.0 - th * th) * math.sqrt(2.0 / math.pi) * (1.0 + 3.0 * 0.044715 * g * g)
    return 0.5 * (1.0 + torch.erf(g * math.sqrt(0.5))) + g * torch.exp(-0.5 * g * g) * math.sqrt(0.5 / math.pi)


def _plain(t):
    case, how = t["case"], t["case"]["how"]
    if how == "norm_fwd":
        out, s = {}, t["X"].float()
        if case["res"]:
            out["S"] = (s + t["R"].float()).to(t["X"].dtype)
            s = out["S"].float()  # the norm of the sum as it is stored
        mean = s.mean(1, keepdim=True)
        d = s - mean
        rstd = torch.rsqrt((d * d).mean(1, keepdim=True) + EPS)
        out["Y"] = (d * rstd * t["gamma"].float() + t["beta"].float()).to(torch.bfloat16)
        out["stats"] = torch.cat((mean, rstd), 1)
        return out
    if how == "norm_bwd":
        mean, rstd = t["stats"][:, :1], t["stats"][:, 1:]
        dy, xh = t["dY"].float(), (t["X"].float() - mean) * rstd
        g = dy * t["gamma"].float()
        dx = rstd * (g - g.mean(1, keepdim=True) - xh * (g * xh).mean(1, keepdim=True))
        if case["res"]:
            dx = dx + t["R"].float()
        return {"dX": dx.to(t["X"].dtype), "dgamma": (dy * xh).sum(0), "dbeta": dy.sum(0)}
    if how == "gated_fwd":
        x = t["X"].float()
        g, u = x @ t["Wg"].float(), x @ t["Wu"].float()
        if case["bias"]:
            g, u = g + t["bg"].float(), u + t["bu"].float()
        out = {"H": (_gate(g, case["act"]) * u).to(torch.bfloat16)}
        if case["save"]:
            out["G"], out["U"] = g.to(torch.bfloat16), u.to(torch.bfloat16)
        return out
    if how == "gated_dact":
        dh = t["dY"].float() @ t["Wd"].float().t() if case["K"] else t["dH"].float()
        g, u = t["G"].float(), t["U"].float()
        return {"dG": (dh * u * _dgate(g, case["act"])).to(torch.bfloat16), "dU": (dh * _gate(g, case["act"])).to(torch.bfloat16)}
    x, dg, du = t["X"].float(), t["dG"].float(), t["dU"].float()
    return {"dX": (dg @ t["Wg"].float().t() + du @ t["Wu"].float().t()).to(torch.bfloat16),
            "dWg": (x.t() @ dg).to(torch.bfloat16), "dWu": (x.t() @ du).to(torch.bfloat16)}


@functools.lru_cache(maxsize=64)
def _plan(T, K, N):
    """The problem statement of a layer and the workspaces that its norm and its gated block want, kept as a program keeps them."""
    import paper_2305_13525_amd as axo

    p = axo.Problem.make((1, 1, 1), (0, 0, 0), T, K, N)
    norm, gated = axo.axo_norm_workspace_bytes(p), axo.axo_gated_workspace_bytes(p)
    return axo, p, torch.zeros(max(norm, 16), dtype=torch.uint8, device=DEV), norm, torch.zeros(max(gated, 16), dtype=torch.uint8, device=DEV), gated


def _ptr(t):
    return None if t is None else t.data_ptr()


def _ld(t):
    return 0 if t is None else t.stride(0)


def _called(t):
    case, how, stream = t["case"], t["case"]["how"], t["stream"]
    if how == "gated_dact":  # the layer behind the block: in-features F, out-features K
        axo, p, _, _, ws, ws_bytes = _plan(case["T"], case["F"], case["K"])
        G, U, dG, dU = t["G"], t["U"], t["dG"], t["dU"]
        if case["K"]:
            axo.axo_gated_dgrad_act(p, t["dY"].data_ptr(), t["dY"].stride(0), t["Wd"].data_ptr(), t["Wd"].stride(0), G.data_ptr(), U.data_ptr(),
                                    G.stride(0), case["act"], dG.data_ptr(), dU.data_ptr(), dG.stride(0), ws.data_ptr(), ws_bytes, stream)
        else:
            axo.axo_gated_dact(p, t["dH"].data_ptr(), t["dH"].stride(0), G.data_ptr(), U.data_ptr(), G.stride(0), case["act"], dG.data_ptr(),
                               dU.data_ptr(), dG.stride(0), stream)
        return {"dG": dG, "dU": dU}
    axo, p, norm_ws, norm_bytes, ws, ws_bytes = _plan(case["T"], case["K"], case["F"])
    X = t["X"]
    if how == "norm_fwd":
        kind, R, S, Y = (axo.AXO_TYPE_F32 if case["wide"] else axo.AXO_TYPE_BF16), t.get("R"), t.get("S"), t["Y"]
        axo.axo_norm_fwd(p, X.data_ptr(), X.stride(0), _ptr(R), _ld(R), kind, t["gamma"].data_ptr(), t["beta"].data_ptr(), EPS, _ptr(S), _ld(S),
                         Y.data_ptr(), Y.stride(0), t["stats"].data_ptr(), stream)
        return {name: t[name] for name in ("S", "Y", "stats") if name in t}
    if how == "norm_bwd":
        kind, R, dY, dX = (axo.AXO_TYPE_F32 if case["wide"] else axo.AXO_TYPE_BF16), t.get("R"), t["dY"], t["dX"]
        axo.axo_norm_bwd(p, dY.data_ptr(), dY.stride(0), X.data_ptr(), X.stride(0), _ptr(R), _ld(R), kind, t["gamma"].data_ptr(),
                         t["stats"].data_ptr(), dX.data_ptr(), dX.stride(0), t["dgamma"].data_ptr(), t["dbeta"].data_ptr(), 0,
                         norm_ws.data_ptr(), norm_bytes, stream)
        return {"dX": dX, "dgamma": t["dgamma"], "dbeta": t["dbeta"]}
    Wg, Wu = t["Wg"], t["Wu"]
    if how == "gated_fwd":
        H, G, U = t["H"], t.get("Gs"), t.get("Us")
        axo.axo_gated_fwd(p, X.data_ptr(), X.stride(0), Wg.data_ptr(), Wu.data_ptr(), Wg.stride(0), _ptr(t.get("bg")), _ptr(t.get("bu")), case["act"],
                          _ptr(G), _ptr(U), _ld(G), H.data_ptr(), H.stride(0), ws.data_ptr(), ws_bytes, stream)
        return {"H": H, "G": G, "U": U} if case["save"] else {"H": H}
    dG, dU, dX, dWg, dWu = t["dG"], t["dU"], t["dX"], t["dWg"], t["dWu"]
    axo.axo_gated_dgrad(p, dG.data_ptr(), dU.data_ptr(), dG.stride(0), Wg.data_ptr(), Wu.data_ptr(), Wg.stride(0), dX.data_ptr(), dX.stride(0),
                        ws.data_ptr(), ws_bytes, stream)
    axo.axo_gated_wgrad(p, X.data_ptr(), X.stride(0), dG.data_ptr(), dU.data_ptr(), dG.stride(0), dWg.data_ptr(), dWu.data_ptr(), dWg.stride(0),
                        ws.data_ptr(), ws_bytes, stream)
    return {"dX": dX, "dWg": dWg, "dWu": dWu}


def run(state):
    return _called(state) if own else _plain(state)


def work(case):
    """Each input read once, each output written once."""
    how, m, k, f = case["how"], case["T"], case["K"], case["F"]
    e = 4.0 if case["wide"] else 2.0
    if how == "norm_fwd":
        return {"bytes": m * k * (e + 2.0 + (2 * e if case["res"] else 0.0)) + 4.0 * k + 8.0 * m, "flops": 8.0 * m * k}
    if how == "norm_bwd":
        return {"bytes": m * k * (2.0 + 2 * e + (e if case["res"] else 0.0)) + 8.0 * m + 10.0 * k, "flops": 14.0 * m * k}
    if how == "gated_fwd":
        out = 3 if case["save"] else 1
        return {"bytes": 2.0 * (m * k + 2.0 * k * f + out * m * f) + (4.0 * f if case["bias"] else 0.0), "flops": 4.0 * m * k * f + 8.0 * m * f}
    if how == "gated_dact":
        return {"bytes": 2.0 * (4.0 * m * f + (m * k + f * k if k else m * f)), "flops": 2.0 * m * k * f + 12.0 * m * f}
    return {"bytes": 2.0 * (2.0 * m * k + 2.0 * m * f + 4.0 * k * f), "flops": 8.0 * m * k * f}


def exact(case, seed):
    t = {name: v.double() for name, v in _inputs(case, seed).items()}
    how, act, m, k = case["how"], case["act"], case["T"], case["K"]

    def gate(z):
        """(act, its derivative) from the derivative of v * P(v): P + v P'."""
        if act == 0:
            prob = torch.sigmoid(z)
            slope = prob * torch.sigmoid(-z)
        elif act == 1:
            inner = math.sqrt(8.0 / math.pi) * (z + 0.044715 * z ** 3)
            prob = torch.sigmoid(inner)
            slope = prob * torch.sigmoid(-inner) * math.sqrt(8.0 / math.pi) * (1.0 + 0.134145 * z ** 2)
        else:
            prob = 0.5 * torch.erfc(-z / math.sqrt(2.0))
            slope = torch.exp(-z ** 2 / 2.0) / math.sqrt(2.0 * math.pi)
        return z * prob, prob + z * slope

    if how == "norm_fwd":
        s = t["X"]
        got = {}
        if case["res"]:
            got["S"] = s + t["R"]
            s = got["S"].to(torch.float32 if case["wide"] else torch.bfloat16).double()
        var, mean = torch.var_mean(s, dim=1, correction=0, keepdim=True)
        rstd = (var + EPS) ** -0.5
        got["Y"] = (s - mean) * rstd * t["gamma"] + t["beta"]
        got["stats"] = torch.cat((mean, rstd), 1)
        return got
    if how == "norm_bwd":
        mean, rstd = t["stats"][:, 0], t["stats"][:, 1]
        xh = (t["X"] - mean.view(m, 1)) * rstd.view(m, 1)
        g = t["dY"] * t["gamma"]
        dx = (g - (g.sum(1) / k).view(m, 1) - xh * ((g * xh).sum(1) / k).view(m, 1)) * rstd.view(m, 1)
        return {"dX": dx + t["R"] if case["res"] else dx, "dgamma": (t["dY"] * xh).sum(0), "dbeta": t["dY"].sum(0)}
    if how == "gated_fwd":
        g, u = torch.mm(t["X"], t["Wg"]), torch.mm(t["X"], t["Wu"])
        if case["bias"]:
            g, u = g + t["bg"], u + t["bu"]
        h = gate(g)[0] * u
        return {"H": h, "G": g, "U": u} if case["save"] else {"H": h}
    if how == "gated_dact":
        dh = torch.mm(t["dY"], t["Wd"].t()) if k else t["dH"]
        value, slope = gate(t["G"])
        return {"dG": dh * t["U"] * slope, "dU": dh * value}
    return {"dX": torch.mm(t["dG"], t["Wg"].t()) + torch.mm(t["dU"], t["Wu"].t()),
            "dWg": torch.mm(t["X"].t(), t["dG"]), "dWu": torch.mm(t["X"].t(), t["dU"])}
