"""A small pre-norm block trained and then answered with, on the library's calls alone where it has one:

    n = norm(x);  o = W2 silu(W1 n);  y = norm(x + o)

Training quantizes the operands of the GEMMs to FP8 / FP4 (the norm delivers its output quantized in both directions, so it is
never stored in bf16), takes the norms' gradients and makes an AdamW step over all four tensors at once: matrices
with 8-bit moments, gains with 32-bit ones, bf16 copies of the matrices for the next step's quantize.  Answering takes a token
of each sequence in bf16 through the same weights in FP4 (snip_gemv).  The activation and the loss are torch's.

    python -m paper_2602_01410_amd.block_example
"""
from __future__ import annotations

import torch
import torch.nn.functional as F

from . import snip

EPS = 1e-5
FP8, FP4, ROW, COL = snip.FP8, snip.FP4, snip.ROW, snip.COL


class Block:
    def __init__(self, dim: int = 512, inner: int = 1024, plan=(FP8, FP8, FP8, FP8, FP8, FP8), seed: int = 0, device="cuda"):
        gen = torch.Generator(device=device).manual_seed(seed)
        self.plan = plan
        master = [torch.randn(inner, dim, generator=gen, device=device) * dim ** -0.5, torch.randn(dim, inner, generator=gen, device=device) * inner ** -0.5,
                  torch.ones(dim, device=device), torch.ones(dim, device=device)]
        # matrices decay and have 8-bit moments and a bf16 copy; gains have none of these
        self.tensors = [snip.alloc_adamw_state(p, torch.empty_like(p, dtype=torch.bfloat16), 8, p.bfloat16(), 0.1) for p in master[:2]]
        self.tensors += [snip.alloc_adamw_state(p, torch.empty_like(p), 32) for p in master[2:]]
        self.step = 0

    def train_step(self, x: torch.Tensor, target: torch.Tensor, lr: float) -> torch.Tensor:
        """One step on x, target (bf16 [tokens, dim], tokens a multiple of 32); returns the loss before it."""
        fx, fw, gdy, gw, wdy, wx = self.plan
        w1, w2, g1, g2 = self.tensors
        (w1r, w1c), (w2r, w2c) = (snip.snip_quantize_both(w.copy, fw, gw) for w in (w1, w2))
        # forward
        n = snip.snip_rms_norm(x, g1.param, EPS, fmt_row=fx, fmt_col=wx)
        a = snip.snip_gemm_fwd(self.plan, n.row, w1r)
        zr, zc = snip.snip_quantize_both(F.silu(a), fx, wx)
        o = snip.snip_gemm_fwd(self.plan, zr, w2r)
        y = snip.snip_rms_norm(o, g2.param, EPS, residual=x)
        diff = y.y.float() - target.float()
        loss = diff.square().mean()
        # backward
        dy = (diff * (2 / diff.numel())).bfloat16()
        dh, g2.grad = snip.snip_rms_norm_backward(dy, y.sum, g2.param, y.rstd)
        dor, doc = snip.snip_quantize_both(dh, gdy, wdy)
        w2.grad = snip.snip_gemm_wgrad(self.plan, doc, zc, out=w2.grad)
        dz = snip.snip_gemm_dgrad(self.plan, dor, w2c).float()
        s = torch.sigmoid(a.float())
        da = (dz * (s + a.float() * s * (1 - s))).bfloat16()
        dar, dac = snip.snip_quantize_both(da, gdy, wdy)
        w1.grad = snip.snip_gemm_wgrad(self.plan, dac, n.col, out=w1.grad)
        dn = snip.snip_gemm_dgrad(self.plan, dar, w1c)
        # (the gradient of x itself, of a block behind another one: dh passes the first norm)
        self.dx, g1.grad = snip.snip_rms_norm_backward(dn, x, g1.param, n.rstd, dsum=dh)
        # update
        self.step += 1
        norm = torch.stack([t.grad.float().square().sum() for t in self.tensors]).sum().sqrt()
        clip = torch.clamp(1.0 / norm, max=1.0).reshape(1)
        snip.snip_adamw_step(self.tensors, lr, 0.9, 0.95, 1e-8, self.step, grad_scale=clip, seed=self.step)
        return loss

    def freeze(self, fmt: int = FP4):
        """The weights to answer with."""
        return [snip.snip_quantize(t.copy, fmt, ROW) for t in self.tensors[:2]]

    def answer(self, x: torch.Tensor, weights) -> torch.Tensor:
        """y of a few tokens (bf16 [tokens, dim])."""
        _, _, g1, g2 = self.tensors
        n = snip.snip_rms_norm(x, g1.param, EPS)
        a, = snip.snip_gemv(n.y, weights[:1])
        o, = snip.snip_gemv(F.silu(a), weights[1:])
        return snip.snip_rms_norm(o, g2.param, EPS, residual=x).y


def train(steps: int = 60, tokens: int = 1024, dim: int = 512, seed: int = 0, lr: float = 2e-3):
    """A student learns what another block of that form answers; returns it, its losses and held-out tokens with their targets."""
    gen = torch.Generator(device="cuda").manual_seed(seed)
    w1, w2 = torch.randn(2 * dim, dim, generator=gen, device="cuda") * dim ** -0.5, torch.randn(dim, 2 * dim, generator=gen, device="cuda") * dim ** -0.5

    def teacher(x):
        h = x.float()
        o = F.silu(F.rms_norm(h, (dim,), eps=EPS) @ w1.t()) @ w2.t()
        return F.rms_norm(h + 2 * o, (dim,), eps=EPS).bfloat16()

    block = Block(dim, 2 * dim, seed=seed + 1)
    losses = []
    for _ in range(steps):
        x = torch.randn(tokens, dim, generator=gen, device="cuda").bfloat16()
        losses.append(block.train_step(x, teacher(x), lr))
    x = torch.randn(8, dim, generator=gen, device="cuda").bfloat16()
    return block, [float(v) for v in losses], x, teacher(x)


if __name__ == "__main__":
    trained, history, held_out, wanted = train(steps=200)
    print("loss of the first and the last steps: %.4f %.4f" % (history[0], sum(history[-10:]) / 10))
    for name, fmt in (("FP8", FP8), ("FP4", FP4)):
        got = trained.answer(held_out, trained.freeze(fmt))
        print("error of answers with %s weights: %.4f" % (name, float((got.float() - wanted.float()).square().mean())))
