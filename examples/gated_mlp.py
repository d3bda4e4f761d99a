"""The MLP half of a transformer block on this library, trained and then asked for single tokens:

    n = norm(x);  h = act(n Wg) * (n Wu);  y = x + h Wd

Training step of one GPU (grid 1 x 1 x 1): axo_norm_fwd, axo_gated_fwd, axo_fc_fwd, then backward axo_fc_wgrad_acc, axo_gated_dgrad_act,
axo_gated_dgrad, axo_gated_wgrad_acc and axo_norm_bwd, which also adds the gradient of the residual.  Activations bf16, master weights and gradients
fp32; torch allocates memory and applies the update (SGD on a clipped gradient).

    python examples/gated_mlp.py --tokens 2048 --width 1024 --inner 2816 --steps 20
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


def _ld(t):
    return t.stride(0)


class GatedMLP:
    """One sublayer: its weights, and the buffers that its passes share."""

    def __init__(self, tokens: int, width: int, inner: int, gate: int = axo.AXO_GATE_SILU, seed: int = 0):
        if width % 8 or inner % 8:
            raise ValueError("rows of multiples of 8 elements")
        self.tokens, self.width, self.inner, self.gate = tokens, width, inner, gate
        gen = torch.Generator(device=DEV)
        gen.manual_seed(seed)
        normal = lambda r, c: torch.empty((r, c), device=DEV).normal_(0.0, 0.02, generator=gen)  # noqa: E731
        self.master = {"gamma": torch.ones(width, device=DEV), "beta": torch.zeros(width, device=DEV), "wg": normal(width, inner), "wu": normal(width, inner),
                       "wd": normal(inner, width)}
        self.grad = {k: torch.zeros_like(v) for k, v in self.master.items()}
        self.w = {k: v.bfloat16() for k, v in self.master.items()}
        bf = lambda r, c: torch.empty((r, c), dtype=torch.bfloat16, device=DEV)  # noqa: E731
        self.n, self.h, self.g, self.u, self.o = bf(tokens, width), bf(tokens, inner), bf(tokens, inner), bf(tokens, inner), bf(tokens, width)
        self.dg, self.du, self.dn, self.dx = bf(tokens, inner), bf(tokens, inner), bf(tokens, width), bf(tokens, width)
        self.stats = torch.empty((tokens, 2), device=DEV)
        self._forwarded = 0  # tokens whose activations the buffers hold for a backward pass
        self._kept = {}  # workspaces of the token counts met so far

    def _plan(self, tokens):
        """The problems of the projections in and out for so many tokens, and the workspaces they want."""
        if tokens not in self._kept:
            up, down = (axo.Problem.make((1, 1, 1), (0, 0, 0), tokens, k, n) for k, n in ((self.width, self.inner), (self.inner, self.width)))
            sizes = (axo.axo_norm_workspace_bytes(up), axo.axo_gated_workspace_bytes(up), axo.axo_gated_workspace_bytes(down))
            self._kept[tokens] = up, down, [(torch.zeros(max(n, 16), dtype=torch.uint8, device=DEV), n) for n in sizes]
        return self._kept[tokens]

    def _check(self, what: str, t: torch.Tensor) -> None:
        """The calls are given addresses: what they read and write has to be there."""
        if t.dtype != torch.bfloat16 or t.dim() != 2 or t.shape[1] != self.width or t.stride(1) != 1 or t.device != self.n.device:
            raise ValueError(f"{what}: rows of {self.width} bfloat16 values on {self.n.device}")
        if t.shape[0] > self.tokens:
            raise ValueError(f"{what}: {t.shape[0]} tokens, and buffers for {self.tokens}")

    def forward(self, x: torch.Tensor, training: bool = True) -> torch.Tensor:
        self._check("x", x)
        m, w, st = x.shape[0], self.w, torch.cuda.current_stream().cuda_stream
        up, down, (_, (ws, nws), _) = self._plan(m)
        self._forwarded = m if training else 0  # n and h are overwritten either way
        save = (self.g.data_ptr(), self.u.data_ptr(), _ld(self.g)) if training else (None, None, 0)
        axo.axo_norm_fwd(up, x.data_ptr(), _ld(x), None, 0, axo.AXO_TYPE_BF16, w["gamma"].data_ptr(), w["beta"].data_ptr(), EPS, None, 0,
                         self.n.data_ptr(), _ld(self.n), self.stats.data_ptr() if training else None, st)
        axo.axo_gated_fwd(up, self.n.data_ptr(), _ld(self.n), w["wg"].data_ptr(), w["wu"].data_ptr(), _ld(w["wg"]), None, None, self.gate, *save,
                          self.h.data_ptr(), _ld(self.h), ws.data_ptr(), nws, st)
        axo.axo_fc_fwd(down, self.h.data_ptr(), _ld(self.h), w["wd"].data_ptr(), _ld(w["wd"]), None, axo.AXO_EPI_NONE, self.o.data_ptr(), _ld(self.o),
                       None, 0, st)
        return x + self.o[:m]

    def backward(self, x: torch.Tensor, dy: torch.Tensor) -> torch.Tensor:
        """Adds the weights' gradients to self.grad and returns x's.  x: of the last forward pass, which was one of training."""
        self._check("x", x)
        self._check("dy", dy)
        if dy.shape != x.shape or x.shape[0] != self._forwarded:
            raise ValueError(f"x has {x.shape[0]} tokens, dy {dy.shape[0]}, and the last forward pass in training had {self._forwarded}")
        w, grad, st = self.w, self.grad, torch.cuda.current_stream().cuda_stream
        up, down, ((wn, nn), (wu, nu), (wd, nd)) = self._plan(x.shape[0])
        axo.axo_fc_wgrad_acc(down, self.h.data_ptr(), _ld(self.h), dy.data_ptr(), _ld(dy), grad["wd"].data_ptr(), _ld(grad["wd"]), None, 0, st)
        axo.axo_gated_dgrad_act(down, dy.data_ptr(), _ld(dy), w["wd"].data_ptr(), _ld(w["wd"]), self.g.data_ptr(), self.u.data_ptr(), _ld(self.g), self.gate,
                                self.dg.data_ptr(), self.du.data_ptr(), _ld(self.dg), wd.data_ptr(), nd, st)
        axo.axo_gated_dgrad(up, self.dg.data_ptr(), self.du.data_ptr(), _ld(self.dg), w["wg"].data_ptr(), w["wu"].data_ptr(), _ld(w["wg"]),
                            self.dn.data_ptr(), _ld(self.dn), wu.data_ptr(), nu, st)
        axo.axo_gated_wgrad_acc(up, self.n.data_ptr(), _ld(self.n), self.dg.data_ptr(), self.du.data_ptr(), _ld(self.dg), grad["wg"].data_ptr(),
                                grad["wu"].data_ptr(), _ld(grad["wg"]), wu.data_ptr(), nu, st)
        axo.axo_norm_bwd(up, self.dn.data_ptr(), _ld(self.dn), x.data_ptr(), _ld(x), dy.data_ptr(), _ld(dy), axo.AXO_TYPE_BF16, w["gamma"].data_ptr(),
                         self.stats.data_ptr(), self.dx.data_ptr(), _ld(self.dx), grad["gamma"].data_ptr(), grad["beta"].data_ptr(), 1, wn.data_ptr(), nn, st)
        return self.dx[:x.shape[0]]

    def update(self, rate: float, most: float = 1.0) -> None:
        """A step along the gradient, which is shortened to a 2-norm of `most` where it is longer."""
        norm = torch.stack([g.square().sum() for g in self.grad.values()]).sum().sqrt()
        scale = -rate * torch.clamp(most / norm, max=1.0)
        for k, v in self.master.items():
            v.add_(self.grad[k] * scale)
            self.w[k].copy_(v)
            self.grad[k].zero_()


def main(argv=None):
    a = argparse.ArgumentParser(description=__doc__, formatter_class=argparse.RawDescriptionHelpFormatter)
    a.add_argument("--tokens", type=int, default=2048)
    a.add_argument("--width", type=int, default=1024)
    a.add_argument("--inner", type=int, default=2816)
    a.add_argument("--steps", type=int, default=20)
    a.add_argument("--rate", type=float, default=0.5)
    args = a.parse_args(argv)
    gen = torch.Generator(device=DEV)
    gen.manual_seed(1)
    x = torch.empty((args.tokens, args.width), device=DEV).normal_(generator=gen).bfloat16()
    teacher, pupil = (GatedMLP(args.tokens, args.width, args.inner, seed=s) for s in (2, 3))
    for k in teacher.w:
        teacher.w[k].mul_(2.0)
    want = teacher.forward(x).float()
    losses = []
    for step in range(args.steps):
        off = pupil.forward(x).float() - want
        losses.append(float(off.square().mean()))
        pupil.backward(x, (off * (2.0 / args.tokens)).bfloat16())
        pupil.update(args.rate)
        print(f"step {step:3d}  loss {losses[-1]:.5f}", flush=True)
    batch = pupil.forward(x, training=False)
    one = pupil.forward(x[-1:], training=False)  # a single token, as when an answer is written
    apart = float((one - batch[-1:]).float().abs().max())
    print(f"a token on its own and in the batch differ by {apart:.4f} at most")
    return losses, apart


if __name__ == "__main__":
    main()
