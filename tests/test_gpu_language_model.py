"""Embedding, losses over the vocabulary and their gradients in one run with the norm, the GEMMs and the optimizer, as block_example.py puts them together."""
import math

import pytest
import torch
import torch.nn.functional as F

from paper_2602_01410_amd import block_example, snip

pytestmark = pytest.mark.gpu
VOCAB, DIM = 1003, 256


def model_and_batch(seed=0, tokens=128):
    model = block_example.LanguageModel(VOCAB, DIM, 512, seed=seed)
    gen = torch.Generator(device="cuda").manual_seed(seed + 1)
    ids, targets = (torch.randint(0, VOCAB, (tokens,), generator=gen, device="cuda") for _ in range(2))
    ids[1] = ids[0]                  # one row twice
    ids[-7:] = -1                    # padding
    targets[-7:] = -100
    return model, ids, targets, gen


def expected(model, ids, loss_of):
    """Loss and gradients by autograd in fp32 on the bf16 weights that the model's calls read."""
    leaves = [(t.copy if t.copy is not None else t.param).float().requires_grad_() for t in model.tensors]
    w1, w2, g1, g2, table = leaves
    x = torch.where((ids >= 0)[:, None], table[ids.clamp(min=0)] * model.scale, 0.0)
    y = F.rms_norm(x + F.silu((F.rms_norm(x, (DIM,), eps=block_example.EPS) * g1) @ w1.t()) @ w2.t(), (DIM,), eps=block_example.EPS) * g2
    loss = loss_of(y @ table.t())
    loss.backward()
    return loss.detach(), [p.grad for p in leaves]


def compare(model, got, loss, grads):
    # FP8's half step is 2^-4 of an element; of the products of a contraction those errors average out, and a few per cent stay (as for the block alone)
    assert abs(float(got) / float(loss) - 1) < 0.02
    for t, want in zip(model.tensors, grads):
        assert float((t.grad.float() - want).norm() / want.norm()) < 0.12


def test_gradients_of_cross_entropy():
    model, ids, targets, _ = model_and_batch()
    got = model.gradients(ids, targets)
    compare(model, got, *expected(model, ids, lambda logits: F.cross_entropy(logits, targets, ignore_index=-100)))


def test_gradients_of_distillation():
    model, ids, _, gen = model_and_batch(3)
    ids[-7:] = 5
    k, tau = 12, 2.0
    indices = torch.stack([torch.randperm(VOCAB, generator=gen, device="cuda")[:k] for _ in ids])
    teacher = torch.randn(len(ids), k, generator=gen, device="cuda") * 3

    def divergence(logits):
        q = torch.softmax(teacher / tau, 1)
        return tau ** 2 * (q * (q.log() - torch.log_softmax(logits / tau, 1).gather(1, indices))).sum(1).mean()
    got = model.distillation_gradients(ids, indices, teacher, tau)
    compare(model, got, *expected(model, ids, divergence))


def test_training_runs():
    model, small, losses, divergences = block_example.train_language_model(steps=3, sequences=2, length=64, vocab=500, dim=256, k=8)
    assert all(math.isfinite(v) for v in losses + divergences) and len(losses) == len(divergences) == 3
    for m in (model, small):
        assert all(torch.isfinite(t.param).all() for t in m.tensors)
        assert torch.equal(m.table.copy, m.table.param.bfloat16())


def test_both_losses_into_one_gradient():
    """Micro-batches add up: the table's gradient of a cross entropy, of a distillation with `accumulate` behind it, and of both embeddings, against 64 bits."""
    gen = torch.Generator(device="cuda").manual_seed(9)
    tokens, vocab, cols, k = 96, 700, 136, 5
    table = (torch.randn(vocab, cols, generator=gen, device="cuda") * 0.2).bfloat16()
    ids, targets = (torch.randint(0, vocab, (tokens,), generator=gen, device="cuda") for _ in range(2))
    at = torch.stack([torch.randperm(vocab, generator=gen, device="cuda")[:k] for _ in range(tokens)])
    teacher = torch.randn(tokens, k, generator=gen, device="cuda")
    x = snip.snip_embed(table, ids)
    assert torch.equal(x, table[ids])
    _, lse = snip.snip_cross_entropy(x, table, targets)
    _, soft = snip.snip_distill(x, table, at, teacher)
    # (one temperature, one lse)
    assert torch.equal(lse, soft)
    dx, dw = snip.snip_cross_entropy_backward(x, table, targets, lse, out_dtype=snip.OUT_FP32)
    dx2, _ = snip.snip_distill_backward(x, table, at, teacher, lse, dw=dw, accumulate=True)
    for d in (dx, dx2):
        snip.snip_embed_backward(d, ids, vocab, dw=dw, accumulate=True)
    X, W = x.double(), table.double()
    p = torch.softmax(X @ W.t(), 1)
    dz = 2 * p
    dz[torch.arange(tokens, device="cuda"), targets] -= 1
    dz.scatter_add_(1, at, -torch.softmax(teacher.double(), 1))
    one = [p.clone(), p.clone()]
    one[0][torch.arange(tokens, device="cuda"), targets] -= 1
    one[1].scatter_add_(1, at, -torch.softmax(teacher.double(), 1))
    want = dz.t() @ X
    want.index_add_(0, ids, dz @ W)
    # each dz is off by 2^-8 (bf16, with 1 % for what fp32 adds) before the products, each dx by 2^-8 again; fp32 sums of at most vocab + tokens terms, a few
    # of them near an element's own cancellation
    half = torch.finfo(torch.bfloat16).eps / 2 * 1.01
    slack = (2 * p + 1e-30) * 2.0 ** -18          # exponentials: an argument up to 32 off by 2^-23, and sums of 136 terms
    err = half * (one[0].abs() + one[1].abs()) + slack
    tol = err.t() @ X.abs()
    rows = err @ W.abs() + half * ((one[0] @ W).abs() + (one[1] @ W).abs() + err @ W.abs())
    tol.index_add_(0, ids, rows)
    mass = (one[0].abs() + one[1].abs())
    tol += (mass.t() @ X.abs() + torch.zeros_like(tol).index_add_(0, ids, mass @ W.abs())) * (vocab + tokens) * 2.0 ** -24
    assert torch.all((dw.double() - want).abs() <= tol), ((dw.double() - want).abs() / tol).max()
