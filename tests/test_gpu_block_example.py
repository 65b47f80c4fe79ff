"""The example that runs the norm, the optimizer and the few-token products together with the GEMMs."""
import pytest
import torch
import torch.nn.functional as F

from paper_2602_01410_amd import block_example, snip

pytestmark = pytest.mark.gpu


def test_training_lowers_the_loss_and_answers_follow_the_weights():
    block, losses, x, target = block_example.train(steps=60)
    assert all(v == v for v in losses)
    assert sum(losses[-5:]) / 5 < 0.6 * losses[0]
    for t in block.tensors[:2]:
        assert torch.equal(t.copy, t.param.bfloat16())
    # answers: the same network in fp32 on the weights that were frozen, up to bf16 between the calls (four roundings of 2^-8)
    for fmt in (snip.FP8, snip.FP4):
        weights = block.freeze(fmt)
        w = []
        for q in weights:
            if fmt == snip.FP8:
                v = q.codes.view(torch.float8_e4m3fn).float()
            else:
                grid = torch.tensor([0, .5, 1, 1.5, 2, 3, 4, 6, 0, -.5, -1, -1.5, -2, -3, -4, -6], device="cuda")
                v = grid[torch.stack((q.codes & 15, q.codes >> 4), 2).long()].reshape(q.rows, q.cols)
            w.append(v * torch.exp2(q.scales.float() - 127).repeat_interleave(32, 1))
        g1, g2 = (t.param for t in block.tensors[2:])
        h = x.float()
        o = F.silu((F.rms_norm(h, h.shape[1:], eps=block_example.EPS) * g1) @ w[0].t()) @ w[1].t()
        want = F.rms_norm(h + o, h.shape[1:], eps=block_example.EPS) * g2
        got = block.answer(x, weights).float()
        assert float((got - want).norm() / want.norm()) < 4 * 2 ** -8
    # the error on held-out tokens stays near the training loss
    err = float((block.answer(x, block.freeze(snip.FP8)).float() - target.float()).square().mean())
    assert err < losses[0]


def test_gradients_of_a_step():
    """dx and the gains' gradients of a step in FP8 against autograd in fp32: the operands' quantization alone is off by a few per cent."""
    block = block_example.Block(256, 512, seed=3)
    gen = torch.Generator(device="cuda").manual_seed(4)
    x, target = (torch.randn(128, 256, generator=gen, device="cuda").bfloat16() for _ in range(2))
    leaves = [t.param.clone().requires_grad_() for t in block.tensors] + [x.float().requires_grad_()]
    w1, w2, g1, g2, h = leaves
    y = F.rms_norm(h + F.silu((F.rms_norm(h, (256,), eps=block_example.EPS) * g1) @ w1.t()) @ w2.t(), (256,), eps=block_example.EPS) * g2
    loss = (y - target.float()).square().mean()
    loss.backward()
    got = block.train_step(x, target, 0.0)
    assert abs(float(got) / float(loss.detach()) - 1) < 0.02
    for mine, leaf in zip([t.grad for t in block.tensors] + [block.dx], leaves):
        assert float((mine.float() - leaf.grad).norm() / leaf.grad.norm()) < 0.12
