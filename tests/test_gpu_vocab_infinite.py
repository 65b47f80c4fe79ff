"""GPU: logits of minus and plus infinity of tokens that take part: entries masked out of the vocabulary, whole tiles of them, entries that the loss names."""
import math

import pytest
import torch

from gpu_util import require_gpu
from test_gpu_vocab_loss import Case, close

pytestmark = pytest.mark.gpu
FAR = -3000.0                                # stands for minus infinity in the reference: its exponential is zero in 64 bits, and differences stay numbers


class Masked(Case):
    """Column 0 of x is 1, or -1 for the tokens `up`; of w it is 0, or minus infinity for the entries `out`.  So those logits are minus infinity, or plus."""

    def __init__(self, tokens, cols, vocab, k, out, up=()):
        super().__init__(tokens, cols, vocab, k, tau=2.0 if k else 1.0, ignored=0.1)
        self.x, self.w = self.x.clone(), self.w.clone()
        self.out = torch.zeros(vocab, dtype=torch.bool, device="cuda")
        self.out[out] = True
        self.up = torch.zeros(tokens, dtype=torch.bool, device="cuda")
        self.up[list(up)] = True
        self.x[:, 0], self.w[:, 0] = 1.0, 0.0
        self.x[self.up, 0] = -1.0
        self.masked = self.w.clone()
        self.masked[self.out, 0] = -math.inf

    def logits(self):
        s, ds = super().logits()
        return torch.where(self.out, FAR, s), torch.where(self.out, 0.0, ds)

    def run(self, snip, **kw):
        finite, self.w = self.w, self.masked
        loss, lse = self.forward(snip)
        dx, dw = self.backward(snip, lse, **kw)
        self.w = finite
        return loss, lse, dx, dw

    def names_out(self):
        """Tokens that name an entry that is masked, and of them those with nothing else."""
        at, q = self.q()
        return (self.out[at] & (q > 0)).any(1)


SHAPES = [(20, 64, 700), (50, 72, 900), (20, 64, 33100), (50, 64, 33100), (100, 72, 1500), (300, 136, 1500), (600, 2056, 33001)]     # every tile
MASKS = {"few": [0, 5, 63, 64, 300, 511], "tiles": [*range(0, 256), *range(320, 384), *range(400, 657)], "most": [*range(0, 200), *range(201, 650)]}


@pytest.mark.parametrize("tokens, cols, vocab", SHAPES)
@pytest.mark.parametrize("k", [0, 4])
@pytest.mark.parametrize("mask", MASKS)
def test_entries_masked_by_minus_infinity(tokens, cols, vocab, k, mask):
    snip = require_gpu()
    out = MASKS[mask] + ([*range(650, vocab - 1)] if mask == "most" else [vocab - 1])
    c = Masked(tokens, cols, vocab, k, out)
    c.at[3], c.at[4] = 0, 5                                      # named, and masked
    loss, lse, dx, dw = c.run(snip)
    wl, we, dl, de = c.want()
    named = c.names_out()
    assert torch.all((lse.double() - we).abs() <= de) and torch.all(loss[named] == math.inf) and named[3] and named[4]
    assert torch.all(((loss.double() - wl).abs() <= dl)[~named])
    (wx, bx), (ww, bw) = c.gradients(lse, c.dloss)
    close(dx[:, 1:], wx[:, 1:], bx[:, 1:])
    close(dw, ww, bw)
    # column 0 of dx is a sum with 0 times infinity in it, of the tokens that take part
    part = c.q()[1].sum(1) > 0
    assert torch.all(torch.isnan(dx[part, 0])) and not dx[~part].any()
    some = torch.ones(vocab, dtype=torch.bool, device="cuda")
    some[c.q()[0][part].flatten()] = False
    assert not dw[c.out & some].any()                            # masked and not named


@pytest.mark.parametrize("tokens, cols, vocab", SHAPES)
@pytest.mark.parametrize("k", [0, 4])
def test_plus_infinity(tokens, cols, vocab, k):
    """log(sum of exponentials) with an infinite one is infinite, and so is the loss, unless it names that one; other tokens are as they were."""
    snip = require_gpu()
    up = [1, 2, 7, tokens - 1]
    c = Masked(tokens, cols, vocab, k, [70, 71, vocab - 2], up)
    c.at[up] = (c.at[up] % 60).to(c.at.dtype)                    # (of a distillation the same number may come twice)
    c.at[2] = 70
    c.at[5] = -100
    c.at[(c.at == 70) & (torch.arange(tokens, device="cuda") != 2).view(-1, *([1] if k else []))] = 1
    loss, lse, dx, dw = c.run(snip)
    wl, we, dl, de = c.want()
    rest = ~c.up
    assert torch.all(lse[c.up] == math.inf) and torch.all((lse.double() - we).abs()[rest] <= de[rest])
    assert torch.isnan(loss[2]) and torch.all(loss[[1, 7, tokens - 1]] == math.inf)
    fine = rest & ~c.names_out()
    assert torch.all((loss.double() - wl).abs()[fine] <= dl[fine])
    # those tokens alone without the others' infinities: the same bits
    d = Masked(tokens, cols, vocab, k, [70, 71, vocab - 2])
    d.x, d.at = torch.where(c.up[:, None], d.x, c.x), c.at
    loss2, lse2, _, _ = d.run(snip)
    assert torch.equal(lse[rest], lse2[rest]) and torch.equal(loss[fine], loss2[fine])
    # dz of those tokens: NaN at the infinite entries, else minus what is wanted
    (wx, bx), _ = c.gradients(lse2, c.dloss)
    close(dx[rest, 1:], wx[rest, 1:], bx[rest, 1:])
    assert torch.all(torch.isnan(dx[c.up])) and torch.all(torch.isnan(dw[[70, 71, vocab - 2]])) and not torch.isnan(dw[~c.out]).any()


def test_nothing_but_minus_infinity():
    """The sum of exponentials is zero: its logarithm is minus infinity, and a loss no number."""
    snip = require_gpu()
    for tokens, vocab in ((20, 300), (300, 515)):
        c = Masked(tokens, 64, vocab, 0, [*range(vocab)])
        c.at[3] = -100
        loss, lse, _, dw = c.run(snip)
        assert torch.all(lse == -math.inf) and loss[3] == 0 and torch.all(torch.isnan(loss[c.at >= 0]))
