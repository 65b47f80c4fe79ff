"""GPU: softmax cross entropy and distillation over a vocabulary, and their gradients, against plain forms in 64 bits."""
import math

import pytest
import torch

from gpu_util import require_gpu

pytestmark = pytest.mark.gpu

HALF32, HALF16 = 2.0 ** -24, 2.0 ** -8       # half a step relative to the value, 2^-p of a significand of p bits: 24 in fp32, 8 in bf16 (torch.finfo(t).eps / 2)


class Case:
    """Inputs of a loss and what it is in 64 bits, with bounds of what rounding may add."""

    def __init__(self, tokens, cols, vocab, k=0, tau=1.0, index=torch.int64, teacher=torch.float32, pad=0, ignored=0.0, seed=0, std=0.3):
        gen = torch.Generator(device="cuda").manual_seed(seed + tokens * 7 + cols + vocab)
        randn = lambda r, c: torch.randn(r, c + pad, generator=gen, device="cuda")  # noqa: E731
        self.x, self.w = randn(tokens, cols).bfloat16()[:, :cols], (randn(vocab, cols) * (std * 8 / math.sqrt(cols))).bfloat16()[:, :cols]
        self.k, self.tau, self.vocab = k, tau, vocab
        n = max(k, 1)
        at = torch.randint(0, vocab, (tokens, n), generator=gen, device="cuda")
        if k and n <= vocab:                 # apart from each other
            at = torch.stack([torch.randperm(vocab, generator=gen, device="cuda")[:n] for _ in range(tokens)]) if tokens else at
        out = torch.rand(tokens, generator=gen, device="cuda") < ignored
        at[out] = -100
        self.at = (at if k else at[:, 0].contiguous()).to(index)
        self.teacher = (torch.randn(tokens, n, generator=gen, device="cuda") * 3).to(teacher) if k else None
        self.dloss = 0.25 + torch.rand(tokens, generator=gen, device="cuda")

    def q(self):
        at = self.at.long().view(self.x.shape[0], -1)
        there = (at >= 0) & (at < self.vocab)
        if not self.k:
            return at * there, there.double()
        u = torch.where(there, self.teacher.double() / self.tau, -math.inf)
        return at * there, torch.softmax(u, 1).nan_to_num(0.0)

    def largest(self):
        """Of the teacher's logits that are finite."""
        if not self.k:
            return torch.zeros(self.x.shape[0], dtype=torch.float64, device="cuda")
        return self.teacher.double().nan_to_num(0.0, 0.0, 0.0).abs().amax(1) / self.tau

    def logits(self):
        """s, and what its rounding may be off by: sums of cols products in fp32 in any order, and the division by tau."""
        x, w = self.x.double(), self.w.double()
        return x @ w.t() / self.tau, (x.abs() @ w.abs().t()) / self.tau * ((self.x.shape[1] + 2) * HALF32)

    def want(self):
        s, ds = self.logits()
        lse = torch.logsumexp(s, 1)
        at, q = self.q()
        sat = s.gather(1, at)
        loss = (torch.xlogy(q, q) + q * (lse[:, None] - sat)).sum(1) * self.tau ** 2
        # exp of a difference (rounded, times a rounded constant, one step of the instruction) and sums of it: 128 terms of a lane or a few joins
        # in turn, and of the tiles
        spread = (s.amax(1) - s.amin(1)).clamp_min(1)
        dlse = ds.amax(1) + (3 * spread + 300 + self.vocab / 128) * HALF32 + (lse.abs() + s.abs().amax(1)) * 2 * HALF32
        u = self.largest()
        dq = (8 + 4 * u + max(self.k, 1)) * HALF32            # relative, of q; absolute, of log q
        dloss = self.tau ** 2 * (dlse + ds.amax(1) + (lse.abs() + s.abs().amax(1) + u + 20) * dq * 2 + 8 * HALF32 * (lse.abs() + s.abs().amax(1)))
        return loss, lse, dloss * 1.1, dlse * 1.1

    def forward(self, snip, **kw):
        if self.k:
            return snip.snip_distill(self.x, self.w, self.at, self.teacher, self.tau, **kw)
        return snip.snip_cross_entropy(self.x, self.w, self.at, **kw)

    def backward(self, snip, lse, **kw):
        kw = {"dloss": self.dloss} | kw
        if self.k:
            return snip.snip_distill_backward(self.x, self.w, self.at, self.teacher, lse, self.tau, **kw)
        return snip.snip_cross_entropy_backward(self.x, self.w, self.at, lse, **kw)

    def gradients(self, lse, dloss=None):
        """dx, dw in 64 bits from this lse, and their bounds before the output's rounding."""
        s, ds = self.logits()
        at, q = self.q()
        g = (torch.ones_like(self.dloss) if dloss is None else dloss).double() * self.tau
        g = torch.where((q.sum(1) > 0) & (g != 0), g, 0.0)[:, None]
        p = torch.exp(s - lse.double()[:, None])
        wanted = torch.zeros_like(p).scatter_add_(1, at, q)
        live = g != 0
        dz = torch.where(live, g * (p - wanted), 0.0)
        # rounded to bf16 once; p off by its argument's error and a few steps, q by its own; two operations
        u = self.largest()[:, None]
        arg = ds + (s - lse.double()[:, None]).abs() * 3 * HALF32 + 4 * HALF32
        err = dz.abs() * HALF16 * 1.01 + torch.where(live, g.abs() * (p * arg * 1.01 + wanted * (8 + 4 * u + max(self.k, 1)) * HALF32 + (p + wanted) * 4 * HALF32), 0.0)
        # fp32 and bf16 have no normal numbers below 2^-126: exponentials, and their products with g, may become zero there
        err = err + torch.where(live, 2.0 ** -125 * (1 + g.abs()), 0.0)
        x, w = torch.where(live, self.x.double(), 0.0), self.w.double()
        rounded = dz.abs() + err
        dx, ex = dz @ w, err @ w.abs() + rounded @ w.abs() * (self.vocab + 64) * HALF32
        dw, ew = dz.t() @ x, err.t() @ x.abs() + rounded.t() @ x.abs() * (self.x.shape[0] + 64) * HALF32
        return (dx, ex * 1.01), (dw, ew * 1.01)


SHAPES = [(1, 8, 1), (1, 64, 100), (2, 72, 255), (7, 512, 1003), (31, 64, 257), (33, 136, 128), (64, 256, 300), (65, 64, 2), (250, 520, 1003), (257, 72, 513), (300, 1024, 4100)]


def close(got, want, bound):
    assert got.dtype in (torch.float32, torch.bfloat16)
    tol = bound + (want.abs() * HALF16 * 1.01 if got.dtype == torch.bfloat16 else want.abs() * HALF32)
    bad = ~((got.double() - want).abs() <= tol)
    assert not bad.any(), (int(bad.sum()), got[bad][:4], want[bad][:4], tol[bad][:4])


def check(snip, c, **kw):
    loss, lse = c.forward(snip)
    wl, we, dl, de = c.want()
    assert torch.all((lse.double() - we).abs() <= de), ((lse.double() - we).abs() / de).max()
    assert torch.all((loss.double() - wl).abs() <= dl), ((loss.double() - wl).abs() / dl).max()
    dx, dw = c.backward(snip, lse, **kw)
    (wx, bx), (ww, bw) = c.gradients(lse, c.dloss)
    close(dx, wx, bx)
    close(dw, ww, bw)
    return loss, lse, dx, dw


@pytest.mark.parametrize("tokens, cols, vocab", SHAPES)
def test_cross_entropy(tokens, cols, vocab):
    check(require_gpu(), Case(tokens, cols, vocab, index=torch.int32 if tokens % 2 else torch.int64, ignored=0.2))


@pytest.mark.parametrize("tokens, cols, vocab, k, tau, teacher", [
    (1, 8, 3, 2, 1.0, torch.float32), (5, 64, 100, 1, 0.5, torch.bfloat16), (33, 72, 300, 16, 2.0, torch.float32), (64, 136, 513, 64, 1.0, torch.bfloat16),
    (70, 64, 1003, 130, 4.0, torch.float32), (258, 264, 700, 7, 1.5, torch.float32), (3, 16, 1100, 1024, 1.0, torch.float32), (2050, 64, 300, 70, 2.0, torch.bfloat16),
    # more entries than the vocabulary has: most come again
    (20, 64, 100, 1024, 1.0, torch.float32), (40, 72, 300, 400, 2.0, torch.bfloat16), (300, 64, 60, 65, 1.0, torch.float32), (17, 64, 1, 33, 1.0, torch.float32)])
def test_distillation(tokens, cols, vocab, k, tau, teacher):
    check(require_gpu(), Case(tokens, cols, vocab, k, tau, torch.int32 if k % 2 else torch.int64, teacher, ignored=0.2))


@pytest.mark.parametrize("tokens, cols, vocab, k", [(40, 64, 20001, 0), (300, 72, 33000, 3), (64, 64, 16384, 0), (129, 64, 16385, 5),
                                                     (70, 72, 140001, 3), (129, 64, 262145, 0), (2500, 72, 140001, 2), (20, 520, 131073, 4)])
def test_pieces_of_the_vocabulary(tokens, cols, vocab, k):
    check(require_gpu(), Case(tokens, cols, vocab, k, ignored=0.1))


@pytest.mark.parametrize("tokens, cols, vocab, k", [(31, 72, 33001, 0), (31, 72, 33001, 9), (50, 136, 40001, 4), (1, 2056, 66001, 0), (20, 2056, 66001, 3), (50, 2056, 66001, 0)])
def test_few_tokens(tokens, cols, vocab, k):
    """Tiles of more rows, where there are many, and weights beyond the last-level cache."""
    check(require_gpu(), Case(tokens, cols, vocab, k, index=torch.int32))


@pytest.mark.parametrize("tokens, cols, vocab, k, ignored", [
    (2048, 72, 300, 0, 0.5), (2049, 72, 300, 3, 0.5), (8192, 64, 130, 0, 0.9), (16390, 64, 33, 2, 0.4), (2100, 64, 257, 0, 1.1), (600, 264, 5000, 5, 0.6), (130, 520, 1003, 0, 0.99)])
def test_tokens_that_are_not_learned(tokens, cols, vocab, k, ignored):
    """Products over the tokens that take part alone, found by every workgroup or by a kernel of its own."""
    c = Case(tokens, cols, vocab, k, ignored=ignored)
    c.dloss[::5] = 0.0
    if ignored < 1:
        c.at[tokens // 3:tokens // 2] = -1                       # a prompt
    check(require_gpu(), c)


def test_long_contraction_and_splits():
    check(require_gpu(), Case(520, 2080, 9001, 4, 2.0))


@pytest.mark.parametrize("k", [0, 5])
def test_large_tiles(k):
    """All products in tiles of 256 x 256, ragged in every extent."""
    check(require_gpu(), Case(600, 2056, 33001, k, ignored=0.1))


@pytest.mark.parametrize("k", [0, 5])
def test_layouts_and_buffers(k):
    """Rows apart, buffers given, a gradient of fp32 added to what is there, each gradient alone, no dloss."""
    snip = require_gpu()
    c = Case(100, 200, 777, k, pad=24, ignored=0.3)
    loss, lse, dx, dw = check(snip, c)
    out = torch.full((777, 208), 5.0, device="cuda")
    dxp = torch.full((100, 216), 5.0, dtype=torch.bfloat16, device="cuda")
    c.backward(snip, lse, dx=dxp[:, :200], dw=out[:, :200], accumulate=True)
    (wx, bx), (ww, bw) = c.gradients(lse, c.dloss)
    close(out[:, :200], ww + 5, bw)
    assert torch.equal(dxp[:, :200], dx) and torch.all(out[:, 200:] == 5) and torch.all(dxp[:, 200:] == 5)
    half = torch.full((777, 200), 0.5, dtype=torch.bfloat16, device="cuda")
    c.backward(snip, lse, dw=half, accumulate=True)
    close(half, ww + 0.5, bw)
    a, none = c.backward(snip, lse, weights=False)
    assert none is None and torch.equal(a, dx)
    none, b = c.backward(snip, lse, inputs=False)
    assert none is None and torch.equal(b, dw)
    _, d32 = c.backward(snip, lse, out_dtype=snip.OUT_FP32)
    close(d32, ww, bw)
    a, b = c.backward(snip, lse, dloss=None)
    (wx, bx), (ww, bw) = c.gradients(lse)
    close(a, wx, bx), close(b, ww, bw)
    one = torch.empty(100, device="cuda")
    assert torch.equal(c.forward(snip, loss=one)[0], loss) and torch.equal(one, loss)


@pytest.mark.parametrize("k, tokens", [(0, 40), (4, 40), (0, 300), (4, 300)])
def test_tokens_that_take_no_part(k, tokens):
    """Whatever is in their x: a token without a target, one whose dloss is zero; others are not touched by it."""
    snip = require_gpu()
    c = Case(tokens, 72, 500, k, ignored=0.0)
    c.at[3] = -100
    c.at[17] = 500
    c.dloss[20] = 0
    loss, lse, dx, dw = check(snip, c)
    assert loss[3] == 0 and loss[17] == 0 and torch.all(dx[[3, 17, 20]] == 0)
    c.x[3], c.x[17, 5], c.x[20] = math.nan, math.inf, -math.inf
    loss2, lse2 = c.forward(snip)
    keep = torch.ones(tokens, dtype=torch.bool, device="cuda")
    keep[[3, 17, 20]] = False
    assert loss2[3] == 0 and loss2[17] == 0 and torch.equal(loss2[keep], loss[keep]) and torch.equal(lse2[keep], lse[keep])
    dx2, dw2 = c.backward(snip, lse2)
    assert torch.equal(dx2, dx) and torch.equal(dw2, dw)
    c.at[:] = -1
    loss, lse = c.forward(snip)
    dx, dw = c.backward(snip, lse)
    assert not loss.any() and not dx.any() and not dw.any()


def test_entries_of_a_teacher():
    """Logits of minus infinity, numbers outside the vocabulary, the same number twice, a NaN."""
    snip = require_gpu()
    c = Case(70, 64, 300, 6)
    c.teacher[1, 2], c.at[2, 4], c.at[3, 1:], c.teacher[4, 1:] = -math.inf, -1, 300, -math.inf
    c.at[5, 3] = c.at[5, 0]
    c.at[6, :] = c.at[6, 0]
    loss, lse, dx, dw = check(snip, c)
    c.teacher[7] = -math.inf                                 # nothing is wanted
    loss, lse, dx, dw = check(snip, c)
    assert loss[7] == 0 and not dx[7].any()
    c.teacher[8, 0] = math.nan
    loss, lse = c.forward(snip)
    assert torch.isnan(loss[8]) and not torch.isnan(loss[torch.arange(70, device="cuda") != 8]).any() and not torch.isnan(lse).any()


def test_one_entry_is_cross_entropy():
    snip = require_gpu()
    c, d = Case(90, 64, 400), Case(90, 64, 400, 1)
    d.x, d.w, d.at, d.dloss = c.x, c.w, c.at[:, None].contiguous(), c.dloss
    a, b = c.forward(snip), d.forward(snip)
    assert torch.equal(a[0], b[0]) and torch.equal(a[1], b[1])
    for p, q in zip(c.backward(snip, a[1]), d.backward(snip, a[1])):
        assert torch.equal(p, q)


def test_large_and_infinite_logits():
    snip = require_gpu()
    c = Case(40, 64, 600, std=60.0)                          # logits of hundreds: most exponentials are zero
    loss, lse, dx, dw = check(snip, c)
    c.x[5] = math.nan
    loss2, _ = c.forward(snip)
    ok = torch.arange(40, device="cuda") != 5
    assert torch.isnan(loss2[5]) and torch.equal(loss2[ok], loss[ok])


@pytest.mark.parametrize("k", [0, 3])
def test_against_differences(k):
    """The loss's change as every element of x, or of w, goes to its next number up or down the gradient."""
    snip = require_gpu()
    c = Case(33, 64, 200, k, 1.0, std=0.1)
    ones = torch.ones(33, device="cuda")
    _, lse = c.forward(snip)
    dx, dw = c.backward(snip, lse, dloss=ones)
    for name, grad, (_, bound) in zip("xw", (dx, dw), c.gradients(lse)):
        at = getattr(c, name)
        ends, tol = [], 0.0
        for sign in (1, -1):
            up = ((at > 0) == (grad * sign > 0)).to(torch.int16) * 2 - 1          # of the magnitude's bits
            moved = (at.contiguous().view(torch.int16) + up).view(torch.bfloat16)
            setattr(c, name, moved)
            loss = c.forward(snip)[0].double()
            ends.append((moved.double(), loss.sum()))
            # along a way on which a token's logits change by d at most the loss differs from its tangent by d^2 / 2 (the second derivative of
            # lse along a direction is a variance); its own error
            step = moved.double() - at.double()
            d = (step @ c.w.double().t() if name == "x" else c.x.double() @ step.t()).abs().amax(1)
            tol = tol + (d ** 2 / 2).sum() + c.want()[2].sum()
        setattr(c, name, at)
        moved = ends[0][0] - ends[1][0]
        want = (moved * grad.double()).sum()
        tol = tol + (moved.abs() * (bound + grad.double().abs() * HALF16)).sum()
        assert (ends[0][1] - ends[1][1] - want).abs() <= tol
        assert want > 4 * tol, (want, tol)


def test_streams_and_graph():
    """Captured and replayed, with other inputs in the same buffers between the replays; two graphs of their own workspaces."""
    snip = require_gpu()
    c, d = Case(70, 136, 900, ignored=0.2), Case(70, 136, 900, 5, 2.0, ignored=0.2)
    other = torch.cuda.Stream()
    other.wait_stream(torch.cuda.current_stream())
    a = c.forward(snip, stream=other)
    a += c.backward(snip, a[1], stream=other)
    torch.cuda.current_stream().wait_stream(other)
    b = c.forward(snip)
    b += c.backward(snip, b[1])
    assert all(torch.equal(p, q) for p, q in zip(a, b))
    graphs = []
    for z in (c, d):
        n = max(z.k, 1)
        ws = [torch.empty(f(70, 136, 900, n), dtype=torch.uint8, device="cuda") for f in (snip.vocab_loss_workspace_bytes, snip.vocab_loss_backward_workspace_bytes)]
        bufs = [torch.empty(70, device="cuda"), torch.empty(70, device="cuda"), torch.empty(70, 136, dtype=torch.bfloat16, device="cuda"), torch.empty(900, 136, device="cuda")]
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            z.forward(snip, loss=bufs[0], lse=bufs[1], workspace=ws[0])
            z.backward(snip, bufs[1], dx=bufs[2], dw=bufs[3], workspace=ws[1])
        graphs.append((z, g, bufs, ws))
    for _ in range(3):
        for z, g, bufs, _ in graphs:
            g.replay()
        torch.cuda.synchronize()
        for z, g, bufs, _ in graphs:
            loss, lse = z.forward(snip)
            dx, dw = z.backward(snip, lse, out_dtype=snip.OUT_FP32)
            assert all(torch.equal(p, q) for p, q in zip(bufs, (loss, lse, dx, dw)))
            z.x.mul_(-0.7)
            z.at.copy_(z.at.roll(1, 0))
        torch.cuda.synchronize()


@pytest.mark.parametrize("tokens, cols, vocab, k", [(1, 72, 300, 0), (33, 136, 1003, 3), (100, 64, 257, 0), (300, 520, 5003, 6), (600, 2056, 33001, 0), (2100, 72, 515, 2)])
def test_workspace_may_hold_anything(tokens, cols, vocab, k):
    """One workspace for calls of other sizes, captured ones among them, with bytes in it that mean "not a number"."""
    snip = require_gpu()
    c = Case(tokens, cols, vocab, k, ignored=0.3)
    n = max(k, 1)
    want = c.forward(snip)
    want += c.backward(snip, want[1])
    ws = torch.empty(max(snip.vocab_loss_workspace_bytes(tokens, cols, vocab, n), snip.vocab_loss_backward_workspace_bytes(tokens, cols, vocab, n)), dtype=torch.uint8, device="cuda")
    bufs = [torch.empty_like(t) for t in want]

    def calls():
        c.forward(snip, loss=bufs[0], lse=bufs[1], workspace=ws)
        c.backward(snip, bufs[1], dx=bufs[2], dw=bufs[3], workspace=ws)
    graphs = []
    for _ in range(2):
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            calls()
        graphs.append(g)
    for run in (calls, graphs[0].replay, graphs[1].replay, graphs[0].replay):
        ws.fill_(255)
        for t in bufs:
            t.fill_(float("nan"))
        run()
        torch.cuda.synchronize()
        assert all(torch.equal(p, q) for p, q in zip(bufs, want))


def test_no_tokens():
    snip = require_gpu()
    c = Case(0, 64, 50)
    loss, lse = c.forward(snip)
    dx, dw = c.backward(snip, lse)
    assert loss.shape == (0,) and dx.shape == (0, 64) and not dw.any()
    dw = torch.ones(50, 64, device="cuda")
    c.backward(snip, lse, dw=dw, accumulate=True)
    assert torch.all(dw == 1)


def test_weights_of_more_than_2_31_elements():
    """The head's last rows lie behind 2^31 elements, in w and in its gradient: each token's target, and a teacher's entries, are there."""
    snip = require_gpu()
    tokens, cols, vocab = 5, 2056, 1048801
    assert vocab * cols > 2 ** 31
    gen = torch.Generator(device="cuda").manual_seed(1)
    w = torch.empty(vocab, cols, dtype=torch.bfloat16, device="cuda")
    for r in range(0, vocab, 1 << 17):
        w[r:r + (1 << 17)] = torch.randn(min(1 << 17, vocab - r), cols, generator=gen, device="cuda") * 0.05
    x = torch.randn(tokens, cols, generator=gen, device="cuda").bfloat16()
    at = torch.tensor([vocab - 1, 7, vocab - 2, vocab - 70000, 1 << 20], device="cuda")
    pieces = [(r, min(r + (1 << 17), vocab)) for r in range(0, vocab, 1 << 17)]
    z = torch.cat([x.double() @ w[a:b].double().t() for a, b in pieces], 1)
    slack = (x.double().abs() @ w[at].double().abs().t()).amax() * ((cols + 2) * HALF32) * 2 + (300 + vocab / 128 + 60) * HALF32
    for k in (0, 3):                     # (token 2 names one entry twice: each counts, with a third)
        index = at if not k else torch.stack((at, at.flip(0), torch.arange(tokens, device="cuda")), 1)
        teacher = torch.zeros(tokens, 3, device="cuda")
        q = torch.zeros(tokens, vocab, dtype=torch.float64, device="cuda").scatter_add_(1, index.view(tokens, -1), torch.full((tokens, max(k, 1)), 1.0 / max(k, 1), dtype=torch.float64, device="cuda"))
        loss, lse = snip.snip_distill(x, w, index, teacher) if k else snip.snip_cross_entropy(x, w, at)
        want = torch.logsumexp(z, 1)
        assert torch.all((lse.double() - want).abs() <= slack)
        assert torch.all((loss.double() - (want - math.log(max(k, 1)) - (q * z).sum(1))).abs() <= 2 * slack + 30 * 8 * HALF32)
        dx, dw = snip.snip_distill_backward(x, w, index, teacher, lse) if k else snip.snip_cross_entropy_backward(x, w, at, lse)
        dz = torch.exp(z - lse.double()[:, None]) - q
        err = dz.abs() * HALF16 * 1.01 + (torch.exp(z - lse.double()[:, None]) + q) * slack + 2.0 ** -125
        wx, bx = 0, 0
        for a, b in pieces:
            wx, bx = wx + dz[:, a:b] @ w[a:b].double(), bx + (err[:, a:b] + dz[:, a:b].abs() * (vocab + 64) * HALF32) @ w[a:b].double().abs()
        close(dx, wx, bx)
        # dw in its first, middle and last rows, and those that are named
        for rows in (slice(0, 300), slice(vocab // 2, vocab // 2 + 300), slice(vocab - 300, vocab), index.flatten()):
            close(dw[rows], dz[:, rows].t() @ x.double(), err[:, rows].t() @ x.double().abs() + dz[:, rows].abs().t() @ x.double().abs() * 80 * HALF32)


def test_widest_pitch():
    """Rows almost 2^22 elements apart: places within a tile just below 2^31 bytes."""
    snip = require_gpu()
    c = Case(260, 72, 300, 2)
    ld = (1 << 22) - 8
    wide = [torch.empty(n * ld, dtype=torch.bfloat16, device="cuda").as_strided((n, 72), (ld, 1)) for n in (260, 300)]
    wide[0].copy_(c.x), wide[1].copy_(c.w)
    a = c.forward(snip)
    a += c.backward(snip, a[1])
    c.x, c.w = wide
    b = c.forward(snip)
    b += c.backward(snip, b[1])
    assert all(torch.equal(p, q) for p, q in zip(a, b))
