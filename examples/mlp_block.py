"""The MLP half of a transformer block on the library's calls: trained with quantized linears and 8-bit checkpoints, then answering token by token.

    x  ->  norm  ->  up (NVFP4)  ->  SwiGLU or GELU  ->  down (NVFP4)  ->  + x

Between the forward and the backward pass of a step a block holds the 4-bit contexts of its two linears, its input and the nonlinearity's
input in 8 bits and two numbers a row; an answer reads the packed weights that the last forward pass left.

    python examples/mlp_block.py [--tokens 2048] [--hidden 512] [--mlp 1024] [--act swiglu] [--norm rms] [--steps 30]
"""
import argparse
import os
import sys
from dataclasses import dataclass

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
import paper_2510_27527_amd as tj  # noqa: E402
from paper_2510_27527_amd import binding as B  # noqa: E402


@dataclass
class Saved:
    """What the backward pass reads."""
    x: object          # Ckpt8, or the tensor itself
    stats: torch.Tensor
    h: object          # Ckpt8, or the tensor itself
    up: tuple          # (Xq, Wq)
    down: tuple

    def bytes(self):
        total = 0
        for t in (self.x, self.stats, self.h, *self.up, *self.down):
            parts = [t] if isinstance(t, torch.Tensor) else [v for v in vars(t).values() if isinstance(v, torch.Tensor)]
            total += sum(p.numel() * p.element_size() for p in parts)
        return total


class MLPBlock:
    """Master parameters in binary32; the linears' weights are cast to bf16 for the forward call, which packs them."""

    def __init__(self, hidden, mlp, act=B.ACT_SWIGLU, norm=B.NORM_RMS, bits8=True, seed=0, outer=B.OUTER_TENSOR, device="cuda"):
        g = torch.Generator(device=device).manual_seed(seed)
        draw = lambda *s: torch.randn(s, generator=g, device=device)
        self.act, self.norm, self.bits8, self.outer = act, norm, bits8, outer
        self.params = {"gamma": torch.ones(hidden, device=device), "up": draw(mlp * (2 if act == B.ACT_SWIGLU else 1), hidden) * hidden ** -0.5,
                       "down": draw(hidden, mlp) * mlp ** -0.5}
        if norm == B.NORM_LAYER:
            self.params["beta"] = torch.zeros(hidden, device=device)
        self.packed = None                     # (up, down) of the last forward pass

    def forward(self, x):
        """x [N, hidden] bf16 -> (block output, Saved)."""
        p, N = self.params, x.shape[0]
        stats = tj.alloc_stats(N, x.device)
        xc = tj.alloc_ckpt8(*x.shape, x.device) if self.bits8 else None
        y = tj.norm_fwd(x, p["gamma"], p.get("beta"), norm=self.norm, stats=stats, ckpt=xc)
        h, *up = tj.linear_fwd(y, p["up"].bfloat16(), outer=self.outer)
        hc = tj.alloc_act_ckpt8(N, p["down"].shape[1], self.act, x.device) if self.bits8 else None
        a = tj.act_fwd(h, self.act, ckpt=hc)
        o, *down = tj.linear_fwd(a, p["down"].bfloat16(), outer=self.outer)
        self.packed = up[1], down[1]
        return o.add_(x), Saved(xc or x, stats, hc or h, tuple(up), tuple(down))

    def backward(self, do, saved, seed):
        """do [N, hidden] bf16 -> (dx, gradients of the parameters)."""
        da, d_down = tj.linear_bwd(do, *saved.down, seed, 1)
        dh = tj.act_bwd(da, saved.h, self.act)
        dy, d_up = tj.linear_bwd(dh, *saved.up, seed, 0)
        dx, d_gamma, d_beta = tj.norm_bwd(dy, saved.x, saved.stats, self.params["gamma"], norm=self.norm)
        grads = {"gamma": d_gamma, "up": d_up, "down": d_down}
        if d_beta is not None:
            grads["beta"] = d_beta
        return dx.add_(do), grads

    def answer(self, x):
        """The block for a few tokens [M, hidden] on the packed weights: bf16 activations, nothing saved."""
        p, (up, down) = self.params, self.packed
        y = tj.norm_fwd(x, p["gamma"], p.get("beta"), norm=self.norm)
        a = tj.act_fwd(tj.gemv(y, up), self.act)
        return tj.gemv(a, down).add_(x)


def train(block, x, target, steps, lr):
    """Adam on the mean square error; returns the losses."""
    optimizer = torch.optim.Adam(block.params.values(), lr=lr)
    losses = []
    for step in range(steps):
        out, saved = block.forward(x)
        err = out.float() - target
        losses.append(float(err.square().mean()))
        _, grads = block.backward((err * (2.0 / err.numel())).bfloat16(), saved, seed=step)
        for name, g in grads.items():
            block.params[name].grad = g.float()
        optimizer.step()
    return losses


def main():
    ap = argparse.ArgumentParser(description=__doc__, formatter_class=argparse.RawDescriptionHelpFormatter)
    ap.add_argument("--tokens", type=int, default=2048)
    ap.add_argument("--hidden", type=int, default=512)
    ap.add_argument("--mlp", type=int, default=1024)
    ap.add_argument("--act", choices=("swiglu", "gelu"), default="swiglu")
    ap.add_argument("--norm", choices=("rms", "layer"), default="rms")
    ap.add_argument("--steps", type=int, default=30)
    ap.add_argument("--lr", type=float, default=3e-3)
    a = ap.parse_args()
    act = B.ACT_SWIGLU if a.act == "swiglu" else B.ACT_GELU
    norm = B.NORM_RMS if a.norm == "rms" else B.NORM_LAYER
    torch.manual_seed(1)
    x = torch.randn(a.tokens, a.hidden, device="cuda").bfloat16()
    target = x.float() + 0.5 * torch.roll(x.float(), 1, 1)
    block = MLPBlock(a.hidden, a.mlp, act, norm)
    losses = train(block, x, target, a.steps, a.lr)
    print("loss %.4f -> %.4f over %d steps" % (losses[0], losses[-1], a.steps))
    kept = {bits8: MLPBlock(a.hidden, a.mlp, act, norm, bits8).forward(x)[1].bytes() for bits8 in (False, True)}
    print("held for the backward pass: %.2f MB with 8-bit checkpoints, %.2f MB without" % (kept[True] / 1e6, kept[False] / 1e6))
    trained, _ = block.forward(x)
    answers = torch.cat([block.answer(x[i:i + 1]) for i in range(8)])
    off = (answers.float() - trained[:8].float()).norm() / trained[:8].float().norm()
    print("eight answers token by token differ from the training pass by %.3f of their size (activations not quantized)" % float(off))


if __name__ == "__main__":
    main()
