"""A stack of gated sublayers on one fp32 residual stream, normed either side of the additions, its matrices trained by the orthogonalised update:

    s_0 = x, n_0 = norm(x)                                  axo_norm_fwd
    h_i = act(n_i Wg) * (n_i Wu)                            axo_gated_fwd
    o_i = h_i Wd;  s_i+1 = s_i + gate rms(o_i),  n_i+1 = norm(s_i+1)     axo_fc_fwd, axo_resnorm_fwd, but for the last sublayer,
    y = s_i + scale h_i Wd                                  axo_fc_add, which adds to the stream in the product's epilogue

and back by axo_fc_add_dact, axo_fc_wgrad_acc, the gated block's backward calls, axo_resnorm_bwd and axo_norm_bwd.  Matrices: momentum, from which axo_ortho forms an update whose
singular values are all about 1.  Vectors: a step along the gradient.  One GPU (grid 1 x 1 x 1); torch allocates memory and adds the updates.

    python examples/residual_stream.py --tokens 2048 --width 1024 --inner 2816 --layers 4 --steps 20
"""
from __future__ import annotations

import argparse
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
import paper_2305_13525_amd as axo  # noqa: E402

DEV = "cuda:0"
EPS = 1e-5
MATRICES = ("wg", "wu", "wd")


def _at(t):
    """Address and leading dimension."""
    return t.data_ptr(), t.stride(0)


class Stream:
    """The stack: weights, their gradients and momenta, and the buffers of a training step on `tokens` tokens."""

    def __init__(self, tokens: int, width: int, inner: int, layers: int, scale: float = 0.5, seed: int = 0):
        if width % 8 or inner % 8 or layers < 1:
            raise ValueError("rows of multiples of 8 elements, and a sublayer at least")
        self.tokens, self.width, self.layers, self.scale = tokens, width, layers, scale
        gen = torch.Generator(device=DEV)
        gen.manual_seed(seed)
        normal = lambda r, c: torch.empty((r, c), device=DEV).normal_(0.0, r ** -0.5, generator=gen)  # noqa: E731
        self.master = []
        for i in range(layers):
            w = {"wg": normal(width, inner), "wu": normal(width, inner), "wd": normal(inner, width), "gamma": torch.ones(width, device=DEV), "beta": torch.zeros(width, device=DEV)}
            if i + 1 < layers:
                w.update(post=torch.ones(width, device=DEV), gate=torch.full((width,), 0.5, device=DEV))
            self.master.append(w)
        self.grad = [{k: torch.zeros_like(v) for k, v in w.items()} for w in self.master]
        self.momentum = [{k: torch.zeros_like(w[k]) for k in MATRICES} for w in self.master]
        self.w = [{k: v.bfloat16() for k, v in w.items()} for w in self.master]
        self.up, self.down = (axo.Problem.make((1, 1, 1), (0, 0, 0), tokens, k, n) for k, n in ((width, inner), (inner, width)))
        bf = lambda c: torch.empty((tokens, c), dtype=torch.bfloat16, device=DEV)  # noqa: E731
        wide = lambda: torch.empty((tokens, width), device=DEV)  # noqa: E731
        self.kept = [{"n": bf(width), "g": bf(inner), "u": bf(inner), "h": bf(inner), "o": bf(width), "s": wide(), "stats": torch.empty((tokens, 4), device=DEV)} for _ in range(layers)]
        self.y, self.ds, self.dg, self.du, self.dn, self.do = wide(), [wide(), wide()], bf(inner), bf(inner), bf(width), bf(width)
        self.update_of = {k: torch.empty_like(self.w[0][k]) for k in MATRICES}
        # a workspace for each purpose: some begin with counters that only their own calls may touch
        sizes = {"gated_up": axo.axo_gated_workspace_bytes(self.up), "gated_down": axo.axo_gated_workspace_bytes(self.down), "norm": axo.axo_norm_workspace_bytes(self.up),
                 "resnorm": axo.axo_resnorm_workspace_bytes(self.up), "add": axo.axo_fc_add_workspace_bytes(self.down), "ortho": max(axo.axo_ortho_workspace_bytes(p) for p in (self.up, self.down))}
        self._forwarded = False  # whether the buffers hold a forward pass
        self._ws = {k: (torch.zeros(max(n, 16), dtype=torch.uint8, device=DEV), n) for k, n in sizes.items()}

    def _space(self, k):
        t, n = self._ws[k]
        return t.data_ptr(), n

    def _check(self, what: str, t: torch.Tensor) -> None:
        """The calls are given addresses: what they read and write has to be there."""
        if t.dtype != torch.float32 or t.shape != (self.tokens, self.width) or t.stride(1) != 1 or t.stride(0) % 4 or t.data_ptr() % 16 or t.device != self.y.device:
            raise ValueError(f"{what}: {self.tokens} rows of {self.width} float32 values on {self.y.device}, each row at a multiple of 16 bytes")

    def forward(self, x: torch.Tensor) -> torch.Tensor:
        self._check("x", x)
        st, f32, layer, rms = torch.cuda.current_stream().cuda_stream, axo.AXO_TYPE_F32, axo.AXO_NORM_LAYER, axo.AXO_NORM_RMS
        w, a = self.w[0], self.kept[0]
        axo.axo_norm_fwd(self.up, *_at(x), None, 0, f32, w["gamma"].data_ptr(), w["beta"].data_ptr(), EPS, None, 0, *_at(a["n"]), a["stats"].data_ptr(), st)
        self._forwarded = True
        s = x
        for i, (w, a) in enumerate(zip(self.w, self.kept)):
            axo.axo_gated_fwd(self.up, *_at(a["n"]), w["wg"].data_ptr(), *_at(w["wu"]), None, None, axo.AXO_GATE_SILU, a["g"].data_ptr(), *_at(a["u"]), *_at(a["h"]),
                              *self._space("gated_up"), st)
            if i + 1 == self.layers:
                axo.axo_fc_add(self.down, *_at(a["h"]), *_at(w["wd"]), None, axo.AXO_EPI_NONE, *_at(s), f32, self.scale, None, 0, *_at(self.y), *self._space("add"), st)
                return self.y
            b, v = self.kept[i + 1], self.w[i + 1]
            axo.axo_fc_fwd(self.down, *_at(a["h"]), *_at(w["wd"]), None, axo.AXO_EPI_NONE, *_at(a["o"]), None, 0, st)
            axo.axo_resnorm_fwd(self.up, *_at(a["o"]), *_at(s), f32, rms, w["post"].data_ptr(), None, w["gate"].data_ptr(), 1.0, layer, v["gamma"].data_ptr(), v["beta"].data_ptr(), EPS,
                                *_at(b["s"]), *_at(b["n"]), b["stats"].data_ptr(), st)
            s = b["s"]

    def backward(self, x: torch.Tensor, dy: torch.Tensor) -> torch.Tensor:
        """Adds the weights' gradients to self.grad and returns x's, which stands until the next call.  x: of the forward pass before."""
        self._check("x", x)
        self._check("dy", dy)
        if not self._forwarded:
            raise ValueError("no forward pass yet")
        st, f32, layer, rms = torch.cuda.current_stream().cuda_stream, axo.AXO_TYPE_F32, axo.AXO_NORM_LAYER, axo.AXO_NORM_RMS
        axo.axo_fc_add_dact(self.down, *_at(dy), f32, None, 0, axo.AXO_EPI_NONE, self.scale, *_at(self.do), st)
        ds = dy
        for i in reversed(range(self.layers)):
            w, g, a = self.w[i], self.grad[i], self.kept[i]
            axo.axo_fc_wgrad_acc(self.down, *_at(a["h"]), *_at(self.do), *_at(g["wd"]), None, 0, st)
            axo.axo_gated_dgrad_act(self.down, *_at(self.do), *_at(w["wd"]), a["g"].data_ptr(), *_at(a["u"]), axo.AXO_GATE_SILU, self.dg.data_ptr(), *_at(self.du),
                                    *self._space("gated_down"), st)
            axo.axo_gated_dgrad(self.up, self.dg.data_ptr(), *_at(self.du), w["wg"].data_ptr(), *_at(w["wu"]), *_at(self.dn), *self._space("gated_up"), st)
            axo.axo_gated_wgrad_acc(self.up, *_at(a["n"]), self.dg.data_ptr(), *_at(self.du), g["wg"].data_ptr(), *_at(g["wu"]), *self._space("gated_up"), st)
            into = self.ds[i % 2]  # the gradient that comes from behind is in the other
            if i == 0:
                axo.axo_norm_bwd(self.up, *_at(self.dn), *_at(x), *_at(ds), f32, w["gamma"].data_ptr(), a["stats"].data_ptr(), *_at(into), g["gamma"].data_ptr(), g["beta"].data_ptr(), 1,
                                 *self._space("norm"), st)
                return into
            b, v, gb = self.kept[i - 1], self.w[i - 1], self.grad[i - 1]
            axo.axo_resnorm_bwd(self.up, *_at(self.dn), *_at(ds), *_at(b["o"]), *_at(a["s"]), f32, rms, v["post"].data_ptr(), None, v["gate"].data_ptr(), 1.0, layer, w["gamma"].data_ptr(),
                                a["stats"].data_ptr(), *_at(into), *_at(self.do), gb["post"].data_ptr(), None, gb["gate"].data_ptr(), g["gamma"].data_ptr(), g["beta"].data_ptr(), 1,
                                *self._space("resnorm"), st)
            ds = into

    def update(self, rate: float, kept: float = 0.9) -> None:
        """A step of `rate` along the orthogonalised momentum of each matrix, and along each vector's gradient; the gradients are cleared."""
        st = torch.cuda.current_stream().cuda_stream
        for master, w, grad, momentum in zip(self.master, self.w, self.grad, self.momentum):
            for k, m in momentum.items():
                m.mul_(kept).add_(grad[k])
                o, p = self.update_of[k], self.down if k == "wd" else self.up
                axo.axo_ortho(p, *_at(m), axo.AXO_TYPE_F32, 5, None, 1e-7, *_at(o), *self._space("ortho"), st)
                master[k].add_(o, alpha=-rate)
            for k in master.keys() - momentum.keys():
                master[k].add_(grad[k], alpha=-rate)
            for k, v in master.items():
                w[k].copy_(v)
                grad[k].zero_()


def main(argv=None):
    a = argparse.ArgumentParser(description=__doc__, formatter_class=argparse.RawDescriptionHelpFormatter)
    a.add_argument("--tokens", type=int, default=2048)
    a.add_argument("--width", type=int, default=1024)
    a.add_argument("--inner", type=int, default=2816)
    a.add_argument("--layers", type=int, default=4)
    a.add_argument("--steps", type=int, default=20)
    a.add_argument("--rate", type=float, default=0.02)
    args = a.parse_args(argv)
    gen = torch.Generator(device=DEV)
    gen.manual_seed(1)
    x = torch.empty((args.tokens, args.width), device=DEV).normal_(generator=gen)
    teacher, pupil = (Stream(args.tokens, args.width, args.inner, args.layers, seed=s) for s in (2, 3))
    want = teacher.forward(x)
    losses = []
    for step in range(args.steps):
        off = pupil.forward(x) - want
        losses.append(float(off.square().mean()))
        pupil.backward(x, off * (2.0 / off.numel()))
        pupil.update(args.rate)
        print(f"step {step:3d}  loss {losses[-1]:.5f}", flush=True)
    return losses


if __name__ == "__main__":
    main()
