"""GPU: gradients of training batches on the large tile in all its forms: several pieces of the vocabulary, so that dx is added to; the head's gradient in fp32, and
added in either type; each with rows apart."""
import pytest
import torch

from gpu_util import require_gpu
from test_gpu_vocab_loss import Case, close

pytestmark = pytest.mark.gpu


def check(c, forms):
    snip = require_gpu()
    loss, lse = c.forward(snip)
    wl, we, dl, de = c.want()
    assert torch.all((lse.double() - we).abs() <= de) and torch.all((loss.double() - wl).abs() <= dl)
    (wx, bx), (ww, bw) = c.gradients(lse, c.dloss)
    vocab, cols = ww.shape
    gen = torch.Generator(device="cuda").manual_seed(3)
    first = None
    for dtype, add in forms:
        whole = torch.randn(vocab, cols + 8, generator=gen, device="cuda").to(dtype)
        before = whole.clone()
        dx, dw = c.backward(snip, lse, dw=whole[:, :cols], accumulate=add)
        close(dx, wx, bx)
        # (what is added to is one more term of the fp32 sum)
        old = before[:, :cols].double() if add else torch.zeros_like(ww)
        close(dw, ww + old, bw + (ww.abs() + bw + old.abs()) * 2.0 ** -24)
        assert torch.equal(whole[:, cols:], before[:, cols:])
        first = dx if first is None else first
        assert torch.equal(dx, first)


ALL = [(torch.bfloat16, False), (torch.float32, False), (torch.bfloat16, True), (torch.float32, True)]


@pytest.mark.parametrize("k", [0, 5])
def test_one_piece(k):
    check(Case(600, 2056, 33001, k, ignored=0.1, pad=8), ALL)


@pytest.mark.parametrize("tokens, cols, vocab, k", [(8200, 264, 33000, 3), (8200, 1032, 70001, 0)])
def test_several_pieces(tokens, cols, vocab, k):
    """Of 32512 entries; dx in seven splits, and in three."""
    check(Case(tokens, cols, vocab, k, ignored=0.1), ALL)
