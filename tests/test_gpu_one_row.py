"""GPU: matrices of one row, whose stride says nothing: the last token of a batch of one, a column that is transposed, a vocabulary of one entry."""
import pytest
import torch

from gpu_util import require_gpu

pytestmark = pytest.mark.gpu

COLS, VOCAB = 64, 200


def rows(kind, cols, dtype=torch.bfloat16):
    """[1, cols] with a stride of its own: of a row, beyond the widest pitch, below the width, odd."""
    empty = lambda *size: torch.empty(size, dtype=dtype, device="cuda")  # noqa: E731
    return {"row": lambda: empty(1, cols), "last": lambda: empty(1, (1 << 22) // cols + 1, cols)[:, -1], "column": lambda: empty(cols, 1).t(),
            "odd": lambda: empty(1, 3 * cols + 5)[:, :cols]}[kind]()


KINDS = ["row", "last", "column", "odd"]


@pytest.mark.parametrize("kind", KINDS)
def test_one_token(kind):
    snip = require_gpu()
    gen = torch.Generator(device="cuda").manual_seed(1)
    w = (torch.randn(VOCAB, COLS, generator=gen, device="cuda") * 0.2).bfloat16()
    ids, targets = torch.tensor([7], device="cuda"), torch.tensor([11], device="cuda")
    at, teacher = torch.tensor([[3, 90, 4]], device="cuda"), torch.tensor([[1.0, 0.5, 2.0]], device="cuda")
    x = rows(kind, COLS)
    assert snip.snip_embed(w, ids, 2.0, out=x) is x and torch.equal(x, w[7:8] * 2)
    plain = w[7:8] * 2
    for loss, back, extra in ((snip.snip_cross_entropy, snip.snip_cross_entropy_backward, (targets,)), (snip.snip_distill, snip.snip_distill_backward, (at, teacher))):
        want = loss(plain, w, *extra)
        got = loss(x, w, *extra)
        assert all(torch.equal(a, b) for a, b in zip(got, want))
        dx, dw = back(plain, w, *extra, want[1])
        out = rows(kind, COLS)
        a, b = back(x, w, *extra, want[1], dx=out)
        assert a is out and torch.equal(a, dx) and torch.equal(b, dw)
    dw = snip.snip_embed_backward(x, ids, VOCAB)
    assert torch.equal(dw[7:8], plain.float()) and torch.count_nonzero(dw) == torch.count_nonzero(plain)


@pytest.mark.parametrize("kind", KINDS)
def test_one_entry(kind):
    snip = require_gpu()
    gen = torch.Generator(device="cuda").manual_seed(2)
    x = torch.randn(30, COLS, generator=gen, device="cuda").bfloat16()
    one, zeros = rows(kind, COLS), torch.zeros(30, dtype=torch.int64, device="cuda")
    one.copy_(x[3:4])
    assert torch.equal(snip.snip_embed(one, zeros), x[3:4].expand(30, COLS))
    want, got = snip.snip_cross_entropy(x, x[3:4].clone(), zeros), snip.snip_cross_entropy(x, one, zeros)
    assert all(torch.equal(a, b) for a, b in zip(got, want))
    # (one entry has all the probability: no gradient)
    for dtype in (torch.bfloat16, torch.float32):
        out = rows(kind, COLS, dtype)
        out.fill_(3.0)
        dx, dw = snip.snip_cross_entropy_backward(x, one, zeros, want[1], dw=out, accumulate=True)
        assert dw is out
        wx, ww = snip.snip_cross_entropy_backward(x, x[3:4].clone(), zeros, want[1], dw=torch.full((1, COLS), 3.0, dtype=dtype, device="cuda"), accumulate=True)
        assert torch.equal(dx, wx) and torch.equal(dw, ww)
        out.fill_(3.0)
        assert torch.equal(snip.snip_embed_backward(x, zeros, 1, dw=out, accumulate=True), snip.snip_embed_backward(x, zeros, 1, dw=torch.full((1, COLS), 3.0, dtype=dtype, device="cuda"), accumulate=True))
