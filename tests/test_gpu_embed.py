"""GPU: rows of an embedding and their gradient against plain sums in 64 bits."""
import pytest
import torch

from gpu_util import require_gpu

pytestmark = pytest.mark.gpu

HALF32, HALF16 = 2.0 ** -24, 2.0 ** -8       # half a step relative to the value, 2^-p of a significand of p bits: 24 in fp32, 8 in bf16 (torch.finfo(t).eps / 2)


def table(rows, cols, ld, dtype, gen, std=1.0):
    return (torch.randn(rows, ld, generator=gen, device="cuda") * std).to(dtype)[:, :cols]


def numbers(n, vocab, dtype, gen, outside=True):
    ids = torch.randint(0, vocab, (n,), generator=gen, device="cuda")
    if outside and n > 2:
        ids[n // 2], ids[n // 3] = -1, vocab
        if dtype == torch.int64:
            ids[0] = 1 << 40
    return ids.to(dtype)


@pytest.mark.parametrize("tokens, cols, vocab, pad, dtype, index, scale", [
    (1, 8, 1, 0, torch.bfloat16, torch.int64, 1.0), (1, 4096, 300, 0, torch.bfloat16, torch.int32, 1.0), (5, 72, 7, 8, torch.float32, torch.int64, 8.485),
    (300, 1032, 1000, 24, torch.bfloat16, torch.int32, 32.1), (2049, 2056, 50, 0, torch.float32, torch.int32, 1.0), (64, 1024, 64, 0, torch.float32, torch.int64, -0.3)])
def test_rows(tokens, cols, vocab, pad, dtype, index, scale):
    snip = require_gpu()
    gen = torch.Generator(device="cuda").manual_seed(tokens + cols)
    w, ids = table(vocab, cols, cols + pad, dtype, gen), numbers(tokens, vocab, index, gen)
    out = torch.full((tokens, cols + 16), 7.0, dtype=torch.bfloat16, device="cuda")
    got = snip.snip_embed(w, ids, scale=scale, out=out[:, :cols])
    there = (ids >= 0) & (ids < vocab)
    # one product in fp32, rounded: the bits
    want = torch.where(there[:, None], w[ids.long().clamp(0, vocab - 1)].float() * scale, 0.0).bfloat16()
    assert torch.equal(got.view(torch.int16), want.view(torch.int16)) and torch.all(out[:, cols:] == 7.0)
    assert torch.equal(snip.snip_embed(w, ids, scale=scale), want)


GRADS = [  # tokens, cols, vocab, pad, out, index, scale, accumulate, what the numbers are
    (1, 8, 1, 0, torch.float32, torch.int64, 1.0, False, "any"), (1, 4096, 300, 0, torch.float32, torch.int32, 2.0, True, "any"),
    (64, 520, 3, 0, torch.float32, torch.int64, 1.0, False, "any"), (65, 520, 3, 8, torch.bfloat16, torch.int64, 1.0, False, "any"),
    (1000, 72, 17, 8, torch.float32, torch.int32, 11.3, False, "any"), (1000, 1032, 5000, 0, torch.float32, torch.int64, 1.0, True, "any"),
    (129, 64, 9, 0, torch.float32, torch.int64, 1.0, False, "one"), (4096, 136, 700, 0, torch.bfloat16, torch.int64, 0.5, True, "text"),
    (5000, 64, 130000, 0, torch.float32, torch.int64, 1.0, False, "text"), (3000, 512, 515, 0, torch.float32, torch.int32, 1.0, False, "runs"),
    (500, 64, 40, 0, torch.float32, torch.int64, 1.0, False, "none"), (0, 64, 40, 0, torch.float32, torch.int64, 1.0, False, "any"),
    (0, 64, 40, 0, torch.float32, torch.int64, 1.0, True, "any"),
    # on both sides of what a workgroup of every token looks through
    (1023, 2056, 3, 0, torch.float32, torch.int32, 1.0, True, "any"), (1024, 4104, 900, 8, torch.bfloat16, torch.int64, 0.7, False, "text"),
    (1024, 520, 9, 0, torch.bfloat16, torch.int64, 1.0, True, "one"), (70, 9000, 9, 0, torch.float32, torch.int64, 1.0, False, "one"), (1025, 520, 9, 0, torch.float32, torch.int64, 1.0, True, "one"),
    (1025, 2056, 3, 24, torch.float32, torch.int32, 1.0, True, "any"), (2500, 1032, 900, 8, torch.bfloat16, torch.int32, 0.7, False, "text"), (2048, 264, 1500, 0, torch.float32, torch.int64, 1.0, True, "text"),
    (2048, 264, 15, 8, torch.bfloat16, torch.int32, 1.0, False, "one"), (2049, 264, 15, 0, torch.float32, torch.int64, 1.0, True, "one"),
    (1025, 72, 4000, 0, torch.float32, torch.int64, 1.0, False, "none")]


@pytest.mark.parametrize("tokens, cols, vocab, pad, out, index, scale, add, kind", GRADS)
def test_gradient(tokens, cols, vocab, pad, out, index, scale, add, kind):
    snip = require_gpu()
    gen = torch.Generator(device="cuda").manual_seed(tokens + cols + vocab)
    dy = table(tokens, cols, cols + pad, torch.bfloat16, gen)
    ids = numbers(tokens, vocab, index, gen)
    if kind == "one":
        ids[:] = vocab - 1
    elif kind == "text":                     # a few numbers have most of the tokens
        ids = ((torch.rand(tokens, generator=gen, device="cuda") ** 6) * vocab).long().clamp(0, vocab - 1).to(index)
    elif kind == "runs":                     # runs that end at, before and behind a multiple of 64 places
        ids = torch.repeat_interleave(torch.arange(9, device="cuda"), torch.tensor([64, 65, 63, 128, 1, 127, 200, 300, 2052], device="cuda"))
        ids = ids[torch.randperm(tokens, generator=gen, device="cuda")].to(index)
    elif kind == "none":
        ids[:] = -1
    whole = torch.randn(vocab, cols + pad, generator=gen, device="cuda").to(out)
    whole[:, cols:] = 7.0
    before, dw = whole[:, :cols].double(), whole[:, :cols]
    got = snip.snip_embed_backward(dy, ids, vocab, scale=scale, dw=dw, accumulate=add)
    there = ((ids >= 0) & (ids < vocab)).nonzero()[:, 0]
    want, size = (before.clone() if add else torch.zeros_like(before)), before.abs() if add else torch.zeros_like(before)
    n = torch.zeros(vocab, dtype=torch.float64, device="cuda")
    rows, at = dy[there].double(), ids[there].long()
    scale32 = torch.tensor(scale, dtype=torch.float32).double().item()
    want.index_add_(0, at, rows * scale32), size.index_add_(0, at, rows.abs() * abs(scale32)), n.index_add_(0, at, torch.ones_like(at, dtype=torch.float64))
    # n additions and the last product with its addition in fp32, each half a step of a partial sum; then the output's rounding
    tol = size * ((n + 1) * HALF32)[:, None] * 1.01 + (want.abs() * HALF16 * 1.01 if out == torch.bfloat16 else 0)
    assert torch.all((got.double() - want).abs() <= tol)
    assert torch.all(whole[:, cols:] == 7.0)
    if add:
        untouched = n == 0
        assert torch.equal(got.double()[untouched], before[untouched])
    else:
        again = snip.snip_embed_backward(dy, ids, vocab, scale=scale, out_dtype=snip.OUT_FP32 if out == torch.float32 else snip.OUT_BF16)
        assert torch.equal(again, got)                      # one order of the sums


@pytest.mark.parametrize("tokens, add", [(5000, False), (1000, False), (1000, True), (2000, True), (5000, True)])
def test_order_of_tokens(tokens, add):
    """Tokens of a number are added in their order, also where many waves look through the numbers: a sum that depends on it."""
    snip = require_gpu()
    dy = torch.zeros(tokens, 8, dtype=torch.bfloat16, device="cuda")
    ids = torch.arange(tokens, device="cuda") % (tokens // 5) + 3
    picked = (ids == tokens // 10).nonzero()[:, 0]
    assert len(picked) == 5
    for t, v in zip(picked.tolist(), [2.0 ** 30, 1.0, 1.0, -2.0 ** 30, 3.0]):
        dy[t] = v                            # in order, in fp32: 2^30 takes up the ones
    got = snip.snip_embed_backward(dy, ids, 1200, dw=torch.zeros(1200, 8, device="cuda"), accumulate=add)
    assert torch.all(got[tokens // 10] == 3.0) and torch.count_nonzero(got) == 8


def test_streams_and_graph():
    snip = require_gpu()
    gen = torch.Generator(device="cuda").manual_seed(5)
    w, ids = table(900, 264, 264, torch.float32, gen), numbers(700, 900, torch.int64, gen)
    dy = table(700, 264, 264, torch.bfloat16, gen)
    dw, y = torch.empty(900, 264, device="cuda"), torch.empty(700, 264, dtype=torch.bfloat16, device="cuda")
    ws = torch.empty(snip.embed_workspace_bytes(700, 264, 900), dtype=torch.uint8, device="cuda")
    other = torch.cuda.Stream()
    other.wait_stream(torch.cuda.current_stream())
    a, b = snip.snip_embed(w, ids, 2.0, stream=other), snip.snip_embed_backward(dy, ids, 900, 2.0, stream=other)
    torch.cuda.current_stream().wait_stream(other)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        snip.snip_embed(w, ids, 2.0, out=y)
        snip.snip_embed_backward(dy, ids, 900, 2.0, dw=dw, workspace=ws)
    for seed in range(3):
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(y, a) and torch.equal(dw, b)
        ids.copy_(numbers(700, 900, torch.int64, torch.Generator(device="cuda").manual_seed(50 + seed)))
        dy.mul_(-0.5)
        a, b = snip.snip_embed(w, ids, 2.0), snip.snip_embed_backward(dy, ids, 900, 2.0)
        torch.cuda.synchronize()


@pytest.mark.parametrize("tokens", [40, 2500])
def test_tables_of_more_than_2_31_elements(tokens):
    """Rows behind 2^31 elements, and a workspace with bytes in it that mean "not a number"."""
    snip = require_gpu()
    vocab, cols = 1048801, 2056
    assert vocab * cols > 2 ** 31
    gen = torch.Generator(device="cuda").manual_seed(tokens)
    table = torch.zeros(vocab, cols, dtype=torch.bfloat16, device="cuda")
    ids = torch.cat((torch.randint(vocab - 500, vocab, (tokens - 3,), generator=gen, device="cuda"), torch.tensor([0, 1 << 20, vocab - 1], device="cuda")))
    rows = torch.unique(ids)
    table[rows] = torch.randn(len(rows), cols, generator=gen, device="cuda").bfloat16()
    assert torch.equal(snip.snip_embed(table, ids), table[ids])
    dy = torch.randn(tokens, cols, generator=gen, device="cuda").bfloat16()
    ws = torch.full((snip.embed_workspace_bytes(tokens, cols, vocab),), 255, dtype=torch.uint8, device="cuda")
    want, size = (torch.zeros(len(rows), cols, dtype=torch.float64, device="cuda").index_add_(0, torch.searchsorted(rows, ids), t) for t in (dy.double(), dy.double().abs()))
    for dtype in (torch.float32, torch.bfloat16):
        dw = torch.full((vocab, cols), float("nan"), dtype=dtype, device="cuda")
        snip.snip_embed_backward(dy, ids, vocab, dw=dw, workspace=ws)
        tol = size * ((tokens + 1) * HALF32) * 1.01 + (want.abs() * HALF16 * 1.01 if dtype == torch.bfloat16 else 0)
        assert torch.all((dw[rows].double() - want).abs() <= tol)
        dw[rows] = 0
        assert not dw.any()
        snip.snip_embed_backward(dy, ids, vocab, dw=dw, accumulate=True, workspace=ws)
        assert torch.all((dw[rows].double() - want).abs() <= tol)
