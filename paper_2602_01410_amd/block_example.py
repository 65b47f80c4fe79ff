"""A small pre-norm block trained and then answered with, on the library's calls alone where it has one:

    n = norm(x);  o = W2 silu(W1 n);  y = norm(x + o)

and, between an embedding and a head of the same weights, as a small language model.

Training quantizes the operands of the GEMMs to FP8 / FP4 (the norm delivers its output quantized in both directions, so it is
never stored in bf16), takes the norms' gradients and makes an AdamW step over all four tensors at once: matrices
with 8-bit moments, gains with 32-bit ones, bf16 copies of the matrices for the next step's quantize.  Answering takes a token
of each sequence in bf16 through the same weights in FP4 (snip_gemv).  The activation and the block's own loss are torch's; the language model's losses
(cross entropy, and a teacher's largest logits) are the library's, whose gradient of the head goes to where the embedding's is added.

    python -m paper_2602_01410_amd.block_example
"""
from __future__ import annotations

import torch
import torch.nn.functional as F

from . import snip

EPS = 1e-5
FP8, FP4, ROW, COL = snip.FP8, snip.FP4, snip.ROW, snip.COL


def update(tensors, lr: float, step: int) -> None:
    """One AdamW step over all tensors, their gradient clipped to a norm of 1."""
    norm = torch.stack([t.grad.float().square().sum() for t in tensors]).sum().sqrt()
    clip = torch.clamp(1.0 / norm, max=1.0).reshape(1)
    snip.snip_adamw_step(tensors, lr, 0.9, 0.95, 1e-8, step, grad_scale=clip, seed=step)


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

    def forward(self, x: torch.Tensor) -> torch.Tensor:
        """y of x (bf16 [tokens, dim], tokens a multiple of 32); keeps what backward needs."""
        fx, fw, _, gw, _, wx = self.plan
        w1, w2, g1, g2 = self.tensors
        (w1r, w1c), (w2r, w2c) = (snip.snip_quantize_both(w.copy, fw, gw) for w in (w1, w2))
        n = snip.snip_rms_norm(x, g1.param, EPS, fmt_row=fx, fmt_col=wx)
        a = snip.snip_gemm_fwd(self.plan, n.row, w1r)
        zr, zc = snip.snip_quantize_both(F.silu(a), fx, wx)
        o = snip.snip_gemm_fwd(self.plan, zr, w2r)
        y = snip.snip_rms_norm(o, g2.param, EPS, residual=x)
        self.kept = x, n, a, zc, y, w1c, w2c
        return y.y

    def backward(self, dy: torch.Tensor) -> torch.Tensor:
        """The weights' gradients (in the tensors), and that of x."""
        _, _, gdy, _, wdy, _ = self.plan
        w1, w2, g1, g2 = self.tensors
        x, n, a, zc, y, w1c, w2c = self.kept
        dh, g2.grad = snip.snip_rms_norm_backward(dy, y.sum, g2.param, y.rstd)
        dor, doc = snip.snip_quantize_both(dh, gdy, wdy)
        w2.grad = snip.snip_gemm_wgrad(self.plan, doc, zc, out=w2.grad)
        dz = snip.snip_gemm_dgrad(self.plan, dor, w2c).float()
        s = torch.sigmoid(a.float())
        da = (dz * (s + a.float() * s * (1 - s))).bfloat16()
        dar, dac = snip.snip_quantize_both(da, gdy, wdy)
        w1.grad = snip.snip_gemm_wgrad(self.plan, dac, n.col, out=w1.grad)
        dn = snip.snip_gemm_dgrad(self.plan, dar, w1c)
        # (dh passes the first norm)
        dx, g1.grad = snip.snip_rms_norm_backward(dn, x, g1.param, n.rstd, dsum=dh)
        return dx

    def train_step(self, x: torch.Tensor, target: torch.Tensor, lr: float) -> torch.Tensor:
        """One step on x, target (bf16 [tokens, dim], tokens a multiple of 32); returns the loss before it."""
        diff = self.forward(x).float() - target.float()
        loss = diff.square().mean()
        self.dx = self.backward((diff * (2 / diff.numel())).bfloat16())
        self.step += 1
        update(self.tensors, lr, self.step)
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


class LanguageModel:
    """A block between an embedding and a head that share their weights: x = sqrt(dim) E[ids], logits = y E^T, which are never stored."""

    def __init__(self, vocab: int = 2000, dim: int = 512, inner: int = 1024, plan=(FP8, FP8, FP8, FP8, FP8, FP8), seed: int = 0, device="cuda"):
        gen = torch.Generator(device=device).manual_seed(seed)
        self.block = Block(dim, inner, plan, seed, device)
        table = torch.randn(vocab, dim, generator=gen, device=device) * dim ** -0.5
        self.table = snip.alloc_adamw_state(table, torch.empty_like(table), 8, table.bfloat16(), 0.1)
        self.tensors = self.block.tensors + [self.table]
        self.scale, self.step = dim ** 0.5, 0

    def hidden(self, ids: torch.Tensor) -> torch.Tensor:
        """What the head multiplies, of ids (int32 or int64 [tokens], tokens a multiple of 32; a number outside the vocabulary is padding)."""
        return self.block.forward(snip.snip_embed(self.table.copy, ids, self.scale))

    def backward(self, ids: torch.Tensor, dy: torch.Tensor) -> None:
        """Behind a loss, which has left the head's part of the table's gradient: that of the block, and the embedding's part added to the table's."""
        snip.snip_embed_backward(self.block.backward(dy), ids, self.table.param.shape[0], self.scale, dw=self.table.grad, accumulate=True)

    def gradients(self, ids: torch.Tensor, targets: torch.Tensor) -> torch.Tensor:
        """Of the mean cross entropy over the tokens that have a target; returns the mean."""
        y = self.hidden(ids)
        loss, lse = snip.snip_cross_entropy(y, self.table.copy, targets)
        vocab = self.table.param.shape[0]
        share = ((targets >= 0) & (targets < vocab)).float()
        share /= share.sum().clamp(min=1)
        dy, _ = snip.snip_cross_entropy_backward(y, self.table.copy, targets, lse, share, dw=self.table.grad)
        self.backward(ids, dy)
        return (loss * share).sum()

    def distillation_gradients(self, ids: torch.Tensor, indices: torch.Tensor, teacher: torch.Tensor, temperature: float = 2.0) -> torch.Tensor:
        """Of the mean divergence from a teacher's largest logits (`teacher` [tokens, k], their numbers in `indices`); returns the mean."""
        y = self.hidden(ids)
        loss, lse = snip.snip_distill(y, self.table.copy, indices, teacher, temperature)
        share = torch.full_like(loss, 1 / len(ids))
        dy, _ = snip.snip_distill_backward(y, self.table.copy, indices, teacher, lse, temperature, share, dw=self.table.grad)
        self.backward(ids, dy)
        return loss.mean()

    def update(self, lr: float) -> None:
        self.step += 1
        update(self.tensors, lr, self.step)


def train_language_model(steps: int = 60, sequences: int = 8, length: int = 128, vocab: int = 2000, dim: int = 512, k: int = 16, seed: int = 0, lr: float = 2e-3):
    """A model learns the next token of sequences in which a token mostly determines it; then a smaller one learns the first one's k largest logits.
    Returns both and their losses."""
    gen = torch.Generator(device="cuda").manual_seed(seed)
    after = torch.randperm(vocab, generator=gen, device="cuda")

    def batch():
        ids = [torch.randint(0, vocab, (sequences,), generator=gen, device="cuda")]
        for _ in range(length):
            other = torch.randint(0, vocab, (sequences,), generator=gen, device="cuda")
            ids.append(torch.where(torch.rand(sequences, generator=gen, device="cuda") < 0.1, other, after[ids[-1]]))
        ids = torch.stack(ids, 1)
        return ids[:, :-1].flatten(), ids[:, 1:].flatten()

    model, small = LanguageModel(vocab, dim, 2 * dim, seed=seed + 1), LanguageModel(vocab, dim // 2, dim, seed=seed + 2)
    losses, divergences = [], []
    for _ in range(steps):
        losses.append(model.gradients(*batch()))
        model.update(lr)
    for _ in range(steps):
        ids, _ = batch()
        # (of a batch this small torch's product and top-k will do)
        logits = (model.hidden(ids) @ model.table.copy.t()).topk(k)
        divergences.append(small.distillation_gradients(ids, logits.indices, logits.values))
        small.update(lr)
    return model, small, [float(v) for v in losses], [float(v) for v in divergences]


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
    _, _, history, divergences = train_language_model(steps=200)
    print("cross entropy of the first and the last steps: %.4f %.4f" % (history[0], sum(history[-10:]) / 10))
    print("divergence of a smaller model from that one: %.4f %.4f" % (divergences[0], sum(divergences[-10:]) / 10))
