"""Host-side checks of the embedding and vocabulary-loss calls: arguments are rejected before any launch (no GPU is needed: the pointers
are never followed), sizes are right and never fall as an extent grows."""
import ctypes

import pytest
import torch

from test_abi import lib

NULL, SHAPE, FORMAT, LAYOUT, WORKSPACE = 1, 2, 3, 4, 5
P = ctypes.c_void_p(0x10000)
at = ctypes.c_void_p


@pytest.fixture(scope="module")
def S():
    return lib()


def test_embed(S):
    def embed(w=P, wd=0, vocab=100, cols=64, ldw=64, ids=P, it=1, tokens=4, scale=1.0, y=P, ldy=64):
        return S._lib().snip_embed(w, wd, vocab, cols, ldw, ids, it, tokens, scale, y, ldy, None)
    assert embed(w=None) == NULL and embed(ids=None) == NULL and embed(y=None) == NULL
    assert embed(wd=2) == FORMAT and embed(it=2) == FORMAT and embed(it=-1) == FORMAT and embed(scale=float("inf")) == FORMAT and embed(scale=float("nan")) == FORMAT
    assert embed(tokens=-1) == SHAPE and embed(vocab=0) == SHAPE and embed(vocab=1 << 31) == SHAPE and embed(cols=60) == SHAPE and embed(cols=0) == SHAPE
    assert embed(cols=1 << 20, ldw=1 << 20, ldy=1 << 20) == SHAPE and embed(ldw=56) == SHAPE and embed(ldy=56) == SHAPE
    assert embed(ldw=68) == LAYOUT and embed(ldy=68) == LAYOUT and embed(w=at(0x10008)) == LAYOUT and embed(y=at(0x10004)) == LAYOUT
    assert embed(ids=at(0x10004)) == LAYOUT and embed(ids=at(0x10002), it=0) == LAYOUT


def test_embed_backward(S):
    def back(dy=P, tokens=100, cols=64, ld=64, ids=P, it=1, vocab=50, scale=1.0, dw=P, dt=1, ldw=64, add=0, ws=P, n=1 << 20):
        return S._lib().snip_embed_backward(dy, tokens, cols, ld, ids, it, vocab, scale, dw, dt, ldw, add, ws, n, None)
    assert back(dy=None) == NULL and back(ids=None) == NULL and back(dw=None) == NULL
    assert back(dt=2) == FORMAT and back(it=2) == FORMAT and back(scale=float("nan")) == FORMAT
    assert back(tokens=-1) == SHAPE and back(tokens=1 << 30) == SHAPE and back(vocab=0) == SHAPE and back(vocab=(1 << 30) + 1) == SHAPE and back(cols=12) == SHAPE and back(ld=32) == SHAPE and back(ldw=32) == SHAPE
    assert back(ld=68) == LAYOUT and back(ldw=68) == LAYOUT and back(dw=at(0x10008)) == LAYOUT and back(ids=at(0x10004)) == LAYOUT and back(ws=at(0x10008)) == LAYOUT
    size = S.embed_workspace_bytes(100, 64, 50)
    assert back(ws=None) == WORKSPACE and back(n=size - 1) == WORKSPACE
    assert size == 256 + 512 + 2 * 2 * 64 * 4                 # places of 51 numbers and of 100 tokens, two blocks' partial sums
    assert S.embed_workspace_bytes(-1, 64, 50) == 0 and S.embed_workspace_bytes(1, 0, 50) == 0 and S.embed_workspace_bytes(1, 64, 0) == 0


def losses(S):
    """Both losses and both directions, by the arguments they share."""
    def args(kw):
        d = dict(x=P, tokens=100, cols=64, ldx=64, w=P, vocab=500, ldw=64, index=P, it=1, teacher=P, tt=1, k=4, tau=1.0, loss=P, lse=P, dloss=P, dx=P, lddx=64, dw=P, dt=0,
                 lddw=64, add=0, ws=P, n=1 << 40) | kw
        ops = [d[v] for v in ("x", "tokens", "cols", "ldx", "w", "vocab", "ldw", "index", "it")]
        top = [d[v] for v in ("teacher", "tt", "k", "tau")]
        return ops, top, [d["loss"], d["lse"], d["ws"], d["n"], None], [d[v] for v in ("lse", "dloss", "dx", "lddx", "dw", "dt", "lddw", "add", "ws", "n")] + [None]

    def ce(**kw):
        o, _, f, _ = args(kw)
        return S._lib().snip_cross_entropy(*o, *f)

    def ce_back(**kw):
        o, _, _, b = args(kw)
        return S._lib().snip_cross_entropy_backward(*o, *b)

    def distill(**kw):
        o, t, f, _ = args(kw)
        return S._lib().snip_distill(*o, *t, *f)

    def distill_back(**kw):
        o, t, _, b = args(kw)
        return S._lib().snip_distill_backward(*o, *t, *b)
    return ce, ce_back, distill, distill_back


def test_losses(S):
    ce, ce_back, distill, distill_back = losses(S)
    for call in (ce, ce_back, distill, distill_back):
        assert call(x=None) == NULL and call(w=None) == NULL and call(index=None) == NULL
        assert call(it=2) == FORMAT and call(it=-1) == FORMAT
        assert call(tokens=-1) == SHAPE and call(tokens=(1 << 21) + 1) == SHAPE and call(vocab=0) == SHAPE and call(vocab=1 << 31) == SHAPE and call(cols=60) == SHAPE
        assert call(cols=0) == SHAPE and call(cols=1 << 20, ldx=1 << 20, ldw=1 << 20) == SHAPE and call(ldx=56) == SHAPE and call(ldw=56) == SHAPE and call(ldx=1 << 22) == SHAPE
        assert call(ldw=1 << 22) == SHAPE
        # logits and inputs beyond what a grid of tiles holds
        assert call(tokens=1 << 21, vocab=(1 << 16) + 1, k=1) == SHAPE and call(tokens=1 << 21, vocab=1 << 16, k=1, ws=None) == WORKSPACE
        assert call(tokens=1 << 20, cols=(1 << 17) + 8, ldx=1 << 18, ldw=1 << 18, lddx=1 << 18, lddw=1 << 18, k=1) == SHAPE
        assert call(ldx=68) == LAYOUT and call(ldw=68) == LAYOUT and call(x=at(0x10008)) == LAYOUT and call(w=at(0x10008)) == LAYOUT and call(index=at(0x10004)) == LAYOUT
        assert call(lse=at(0x10002)) == LAYOUT and call(ws=at(0x10008)) == LAYOUT
        assert call(ws=None) == WORKSPACE and call(n=1000) == WORKSPACE
    for call in (ce, distill):
        assert call(loss=None, lse=None) == NULL and call(loss=at(0x10002)) == LAYOUT
        assert call(tokens=0, x=None, index=None, teacher=None, ws=None, n=0) == 0
    for call in (ce_back, distill_back):
        assert call(lse=None) == NULL and call(dx=None, dw=None) == NULL and call(dt=2) == FORMAT
        assert call(dx=at(0x10008)) == LAYOUT and call(lddx=68) == LAYOUT and call(lddx=56) == SHAPE and call(dw=at(0x10008)) == LAYOUT and call(lddw=68) == LAYOUT
        assert call(lddw=56) == SHAPE and call(dloss=at(0x10002)) == LAYOUT
    for call in (distill, distill_back):
        assert call(teacher=None) == NULL and call(tt=2) == FORMAT and call(teacher=at(0x10002)) == LAYOUT and call(teacher=at(0x10001), tt=0) == LAYOUT
        assert call(k=0) == SHAPE and call(k=1025) == SHAPE and call(tokens=1 << 21, k=1024) == SHAPE
        for tau in (0.0, -1.0, float("nan"), float("inf"), 1e-39, 1e-19, 1.9e19, -2.0):
            assert call(tau=tau) == FORMAT
        assert call(tau=1.1e-19, ws=None) == WORKSPACE and call(tau=1.8e19, ws=None) == WORKSPACE


@pytest.mark.parametrize("name, extents", [
    ("embed_workspace_bytes", ([0, 1, 63, 64, 65, 4096, 100000], [8, 64, 4096, 8192], [1, 15, 16, 500, 128000])),
    ("vocab_loss_workspace_bytes", ([0, 1, 31, 32, 33, 63, 64, 65, 128, 129, 255, 256, 257, 300, 4096, 16384, 65536], [8, 4096], [1, 127, 128, 129, 257, 16384, 16385, 128000],
                                    [1, 2, 4, 5, 64, 1024])),
    ("vocab_loss_backward_workspace_bytes", ([0, 1, 31, 32, 33, 63, 64, 65, 128, 129, 255, 256, 257, 300, 1000, 4096, 4097, 8192, 16384, 16385, 40000, 65536],
                                             [8, 64, 512, 2048, 4096, 8192], [1, 100, 255, 256, 257, 511, 512, 513, 1024, 4096, 4097, 8192, 16384, 16385, 32000, 128000],
                                             [1, 2, 4, 5, 64]))])
def test_workspaces_grow(S, name, extents):
    """One for a program's largest call serves the smaller ones."""
    import itertools
    size = getattr(S, name)
    for point in itertools.product(*extents):
        here = size(*point)
        for d, values in enumerate(extents):
            i = values.index(point[d])
            if i + 1 < len(values):
                assert here <= size(*point[:d], values[i + 1], *point[d + 1:]), (point, d)


def test_workspace_is_enough(S):
    """A call takes no more than the size that is asked for: sizes just short of it may do, the size itself is never refused (an absent gradient
    buffer is what is noticed first)."""
    ce, ce_back, distill, distill_back = losses(S)
    for tokens in (1, 40, 64, 65, 300, 4096, 20000, 70000):
        for cols in (8, 520, 4096):
            for vocab in (1, 300, 5000, 16385, 128000):
                for k in (1, 3, 64):
                    n, m = S.vocab_loss_workspace_bytes(tokens, cols, vocab, k), S.vocab_loss_backward_workspace_bytes(tokens, cols, vocab, k)
                    kw = dict(tokens=tokens, cols=cols, vocab=vocab, k=k, ldx=cols, ldw=cols, lddx=cols, lddw=cols, ws=at(0x10008))
                    # the workspace is looked at last: its size first, then its alignment
                    assert distill(n=n, **kw) == LAYOUT and distill_back(n=m, **kw) == LAYOUT and distill(n=n // 4, **kw) == WORKSPACE


def test_binding_refuses(S):
    """Without a GPU: what is no CUDA tensor is refused by name before anything else."""
    x = torch.zeros(4, 64, dtype=torch.bfloat16)
    ids = torch.zeros(4, dtype=torch.int64)
    ws = torch.zeros(16, dtype=torch.uint8)
    for call in (lambda: S.snip_embed(x, ids, out=x), lambda: S.snip_embed_backward(x, ids, 4, dw=x, workspace=ws),
                 lambda: S.snip_cross_entropy(x, x, ids, loss=x, lse=x, workspace=ws), lambda: S.snip_distill_backward(x, x, ids, x, x, dx=x, dw=x, workspace=ws)):
        with pytest.raises((ValueError, RuntimeError)):
            call()
    with pytest.raises(ValueError, match="accumulate"):
        S.snip_embed_backward(x, ids, 4, accumulate=True)
    with pytest.raises(ValueError, match="rows"):
        S.snip_embed_backward(x, ids, 5, dw=x)
    with pytest.raises(ValueError, match="without the gradient"):
        S.snip_cross_entropy_backward(x, x, ids, x, dw=x, weights=False)
    with pytest.raises(ValueError, match="accumulate"):
        S.snip_cross_entropy_backward(x, x, ids, x, accumulate=True)
    with pytest.raises(ValueError, match="teacher"):
        S.snip_distill(x, x, ids, None)
