"""GPU: logits far from zero, as the smallest temperatures make them: the losses are as exact as fp32 holds them, up to its largest numbers."""
import pytest
import torch

from gpu_util import require_gpu
from test_gpu_vocab_loss import Case

pytestmark = pytest.mark.gpu

SHAPES = [(20, 64, 700), (50, 72, 900), (20, 64, 33100), (50, 64, 33100), (100, 72, 1500), (300, 136, 1500), (600, 2056, 33001)]     # every tile


def check(c):
    loss, lse = c.forward(require_gpu())
    wl, we, dl, de = c.want()
    assert torch.all((lse.double() - we).abs() <= de) and torch.all((loss.double() - wl).abs() <= dl)
    return loss, lse


@pytest.mark.parametrize("tokens, cols, vocab", SHAPES)
@pytest.mark.parametrize("tau", [1e-4, 1e-7, 3e-9, 1e-9, 1e-12, 1e-18])
def test_temperatures(tokens, cols, vocab, tau):
    check(Case(tokens, cols, vocab, 4, tau, ignored=0.1))


@pytest.mark.parametrize("tokens, cols, vocab", SHAPES)
@pytest.mark.parametrize("scale", [2.0 ** 20, 2.0 ** 30, 2.0 ** 31, 2.0 ** 40, 2.0 ** 100])
def test_cross_entropy(tokens, cols, vocab, scale):
    c = Case(tokens, cols, vocab, ignored=0.1)
    c.x = c.x * scale
    check(c)
    # no number stays none, beside logits as large
    c.w[vocab // 3] = float("nan")
    loss, lse = c.forward(require_gpu())
    assert torch.all(torch.isnan(lse)) and torch.all(torch.isnan(loss) == (c.at >= 0))


def test_all_far_below_zero():
    """The largest of them is far from zero too."""
    c = Case(40, 64, 600)
    c.x, c.w = c.x.abs() * 2.0 ** 40, -c.w.abs()
    check(c)
