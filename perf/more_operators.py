"""The operators at both ends of a language model, as a program calls them: rows of the embedding in (and their gradient, summed over the
tokens in sorted order), the loss over the vocabulary out: softmax cross entropy, or distillation from a teacher's top logits, each with
its gradients and without keeping the logits.

`run` computes them with elementary torch operations in 32 bits, or, where `own` is set, with the calls of
`paper_2602_01410_amd.snip`.
"""
from __future__ import annotations

import math

import torch

own = False

MOST = 1 << 40              # products of a drawn case: tokens x hidden x vocabulary


def listed():
    return [
        # generation, one token of one sequence: launches are all there is
        {"name": "embed_1x4096", "kind": "embed", "tokens": 1, "cols": 4096, "vocab": 32000, "table": "bf16", "index": "int64", "scale": 1.0},
        # a training batch out of fp32 master weights, rows scaled by the root of their width
        {"name": "embed_16384x4096", "kind": "embed", "tokens": 16384, "cols": 4096, "vocab": 128000, "table": "fp32", "index": "int64", "scale": 64.0},
        # its gradient: an odd batch over an odd vocabulary, added to what is there (a second micro-batch, or a table that is the head too)
        {"name": "embed_grad_1003x2056", "kind": "embed_grad", "tokens": 1003, "cols": 2056, "vocab": 50257, "out": "fp32", "add": True, "index": "int32", "scale": 1.0},
        # a training step of a 7B-shaped model, all of the gradient anew
        {"name": "embed_grad_16384x4096", "kind": "embed_grad", "tokens": 16384, "cols": 4096, "vocab": 32000, "out": "fp32", "add": False, "index": "int64", "scale": 64.0},
        # scoring a short answer with a small model
        {"name": "ce_7x512_1003", "kind": "ce", "tokens": 7, "cols": 512, "vocab": 1003, "index": "int64", "ignored": 0.0},
        # evaluation: 7B-shaped hidden states against a large vocabulary
        {"name": "ce_8192x4096_128000", "kind": "ce", "tokens": 8192, "cols": 4096, "vocab": 128000, "index": "int64", "ignored": 0.02},
        # fine-tuning on a short dialogue, whose prompt is not learned
        {"name": "ce_grad_250x2080_50257", "kind": "ce_grad", "tokens": 250, "cols": 2080, "vocab": 50257, "index": "int64", "ignored": 0.4},
        # a training step of a 7B-shaped model
        {"name": "ce_grad_8192x4096_32000", "kind": "ce_grad", "tokens": 8192, "cols": 4096, "vocab": 32000, "index": "int64", "ignored": 0.02},
        # how far a quantized 1B-shaped student is from its teacher, over a few tokens and over an evaluation batch
        {"name": "distill_37x2048_32000_k8", "kind": "distill", "tokens": 37, "cols": 2048, "vocab": 32000, "k": 8, "teacher": "fp32", "index": "int32", "tau": 2.0, "ignored": 0.0},
        {"name": "distill_4096x2048_128000_k64", "kind": "distill", "tokens": 4096, "cols": 2048, "vocab": 128000, "k": 64, "teacher": "bf16", "index": "int64", "tau": 1.0, "ignored": 0.02},
        # its training steps: a small odd one, and a 1B-shaped one
        {"name": "distill_grad_515x1024_8191_k16", "kind": "distill_grad", "tokens": 515, "cols": 1024, "vocab": 8191, "k": 16, "teacher": "fp32", "index": "int64", "tau": 1.0, "ignored": 0.1},
        {"name": "distill_grad_4096x2048_32000_k32", "kind": "distill_grad", "tokens": 4096, "cols": 2048, "vocab": 32000, "k": 32, "teacher": "bf16", "index": "int32", "tau": 2.0, "ignored": 0.02},
    ]


def _log_int(rng, lo, hi):
    return max(lo, min(hi, round(math.exp(rng.uniform(math.log(lo), math.log(hi + 0.5))))))


def _to8(v):
    return max(8, (v + 4) // 8 * 8)


def draw(rng):
    kind = rng.choice(("embed", "embed_grad", "ce", "ce_grad", "distill", "distill_grad"))
    cols = _to8(_log_int(rng, 64, 4096))
    vocab = _log_int(rng, 100, 128000)
    index = rng.choice(("int64", "int64", "int32"))
    if kind == "embed":
        return {"kind": kind, "tokens": _log_int(rng, 1, 16384), "cols": cols, "vocab": vocab, "table": rng.choice(("bf16", "fp32")), "index": index,
                "scale": rng.choice((1.0, cols ** 0.5))}
    if kind == "embed_grad":
        # (the largest listed one has 128 M elements of gradient)
        return {"kind": kind, "tokens": _log_int(rng, 1, 16384), "cols": cols, "vocab": min(vocab, (1 << 27) // cols), "out": rng.choice(("fp32", "fp32", "bf16")),
                "add": rng.random() < 0.4, "index": index, "scale": rng.choice((1.0, cols ** 0.5))}
    c = {"kind": kind, "tokens": _log_int(rng, 1, min(8192, MOST // (cols * vocab))), "cols": cols, "vocab": vocab, "index": index,
         "ignored": rng.choice((0.0, 0.02, 0.4))}
    if kind.startswith("distill"):
        c |= {"k": min(_log_int(rng, 1, 64), vocab), "teacher": rng.choice(("fp32", "bf16")), "tau": rng.choice((1.0, 2.0, 0.5))}
    return c


def work(case):
    kind, t, c, v = case["kind"], case["tokens"], case["cols"], case["vocab"]
    ids = t * (8 if case["index"] == "int64" else 4)
    if kind == "embed":
        return {"bytes": t * c * ((4 if case["table"] == "fp32" else 2) + 2) + ids, "flops": t * c}
    if kind == "embed_grad":
        # what is added to is read and written only where a token is; new gradients are written whole
        size = 4 if case["out"] == "fp32" else 2
        return {"bytes": t * c * 2 + ids + (2 * size * c * min(t, v) if case["add"] else size * c * v), "flops": t * c}
    if kind.startswith("distill"):
        ids = ids * case["k"] + t * case["k"] * (4 if case["teacher"] == "fp32" else 2)
    operands = 2 * c * (t + v)
    if kind.endswith("_grad"):
        # the logits, formed anew, and two products of that size
        return {"bytes": 2 * operands + ids + 8 * t, "flops": 6 * t * c * v}
    return {"bytes": operands + ids + 8 * t, "flops": 2 * t * c * v}


# ---- inputs ---------------------------------------------------------------------------------------------------------------


def _normed(gen, rows, cols):
    """Hidden states behind a norm: rows of unit variance, one column in a hundred an outlier column."""
    t = torch.randn(rows, cols, generator=gen, device="cuda")
    t *= 1 + 7 * (torch.rand(cols, generator=gen, device="cuda") < 0.01)
    return t.bfloat16()


def _table(gen, vocab, cols, dtype, std):
    t = torch.empty(vocab, cols, dtype=dtype, device="cuda")
    for part in t.split(max(1, (1 << 27) // cols)):
        part.copy_(torch.randn(part.shape, generator=gen, device="cuda") * std)
    return t


def _tokens(gen, n, vocab, dtype):
    """Token numbers as text has them: the r-th most frequent about 1 / r as often as the first, numbers not in order of frequency."""
    u = torch.rand(n, generator=gen, device="cuda", dtype=torch.float64)
    rank = (torch.exp(u * math.log(vocab + 1)) - 1).long().clamp_(0, vocab - 1)
    return (torch.randperm(vocab, generator=gen, device="cuda")[rank]).to(dtype)


def prepare(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    kind, t, c, v = case["kind"], case["tokens"], case["cols"], case["vocab"]
    itype = torch.int64 if case["index"] == "int64" else torch.int32
    s = {"case": case}
    if kind == "embed":
        s["w"] = _table(gen, v, c, torch.float32 if case["table"] == "fp32" else torch.bfloat16, 0.02)
        s["ids"] = _tokens(gen, t, v, itype)
        s["y"] = torch.empty(t, c, dtype=torch.bfloat16, device="cuda")
        if t > 8:
            s["ids"][t // 2] = -1             # a padding token: no row
        return s
    if kind == "embed_grad":
        s["dy"] = (_normed(gen, t, c).float() * 1e-3).bfloat16()
        s["ids"] = _tokens(gen, t, v, itype)
        if t > 8:
            s["ids"][t // 2] = -1
        dtype = torch.float32 if case["out"] == "fp32" else torch.bfloat16
        s["dw"] = _table(gen, v, c, dtype, 1e-3)
        if own:
            _scratch(s)
        return s
    s["x"] = _normed(gen, t, c)
    s["w"] = _table(gen, v, c, torch.bfloat16, 0.02)
    out = torch.rand(t, generator=gen, device="cuda") < case["ignored"]
    if kind.startswith("ce"):
        s["targets"] = _tokens(gen, t, v, itype)
        s["targets"][out] = -100
    else:
        k = case["k"]
        # logits of another model: the largest ones lie close together, the rest falls off
        s["teacher"] = (12 - 2.5 * torch.log1p(torch.arange(k, device="cuda")) + 0.7 * torch.randn(t, k, generator=gen, device="cuda")).to(
            torch.float32 if case["teacher"] == "fp32" else torch.bfloat16)
        first = _tokens(gen, t, v, torch.int64)
        # k numbers apart from each other: steps of an odd size that the vocabulary's size does not divide into fewer than k
        step = v // k
        s["indices"] = ((first[:, None] + torch.arange(k, device="cuda") * step + torch.randint(0, max(1, step), (t, k), generator=gen, device="cuda")) % v).to(itype)
        s["indices"][out] = -100
        if k > 2:
            s["indices"][t // 3, k - 1] = -1                          # fewer logits than k
    s["loss"], s["lse"] = torch.empty(t, device="cuda"), torch.empty(t, device="cuda")
    if kind.endswith("_grad"):
        tau = case.get("tau", 1.0)
        wide = s["w"].float().t()
        for first in range(0, t, 1024):
            s["lse"][first:first + 1024] = torch.logsumexp((s["x"][first:first + 1024].float() @ wide) / tau, 1)
        del wide
        # the mean over tokens, each with a weight of its own
        s["dloss"] = (0.5 + torch.rand(t, generator=gen, device="cuda")) / t
        s["dx"], s["dw"] = torch.empty_like(s["x"]), torch.empty_like(s["w"])
    if own:
        _scratch(s)
    return s


# ---- plain forms ----------------------------------------------------------------------------------------------------------


def _embed(s):
    ids = s["ids"].long()
    there = (ids >= 0) & (ids < s["case"]["vocab"])
    rows = s["w"][ids.clamp(0, s["case"]["vocab"] - 1)].float() * s["case"]["scale"]
    return torch.where(there[:, None], rows, 0.0).bfloat16()


def _embed_grad(s):
    case = s["case"]
    ids = s["ids"].long()
    there = ((ids >= 0) & (ids < case["vocab"])).nonzero().squeeze(1)
    total = torch.zeros(case["vocab"], case["cols"], device="cuda")
    total.index_add_(0, ids[there], s["dy"][there].float())
    total *= case["scale"]
    if case["add"]:
        total += s["dw"].float()
    s["dw"].copy_(total)
    return s["dw"]


def _picked(s):
    """Of each token: the entries of the vocabulary that its loss names, which of them count, and the probabilities they should have."""
    case = s["case"]
    if case["kind"].startswith("ce"):
        index = s["targets"].long()[:, None]
        there = (index >= 0) & (index < case["vocab"])
        return index.clamp(0, case["vocab"] - 1), there, there.float()
    index = s["indices"].long()
    there = (index >= 0) & (index < case["vocab"])
    u = torch.where(there, s["teacher"].float() / case["tau"], -math.inf)
    top = u.amax(1, keepdim=True)
    e = torch.where(there, torch.exp(u - torch.where(top == -math.inf, 0.0, top)), 0.0)
    total = e.sum(1, keepdim=True)
    return index.clamp(0, case["vocab"] - 1), there, torch.where(total > 0, e / total, 0.0)


def _loss(s):
    tau = s["case"].get("tau", 1.0)
    z = (s["x"].float() @ s["w"].float().t()) / tau
    top = z.amax(1, keepdim=True)
    lse = torch.log(torch.exp(z - top).sum(1)) + top[:, 0]
    index, there, q = _picked(s)
    at = z.gather(1, index)
    entropy = torch.where(q > 0, q * torch.log(torch.where(q > 0, q, 1.0)), 0.0)
    loss = (entropy + q * (lse[:, None] - at)).sum(1) * tau ** 2
    return {"loss": torch.where(there.any(1), loss, 0.0), "lse": lse}


def _loss_grad(s):
    tau = s["case"].get("tau", 1.0)
    x, w = s["x"].float(), s["w"].float()
    index, there, q = _picked(s)
    g = s["dloss"] * tau * there.any(1)
    dz = torch.exp((x @ w.t()) / tau - s["lse"][:, None])
    dz.scatter_add_(1, index, -q)
    dz *= g[:, None]
    return {"dx": (dz @ w).bfloat16(), "dw": (dz.t() @ x).bfloat16()}


# ---- the framework's calls ------------------------------------------------------------------------------------------------


def _scratch(s):
    if "scratch" not in s:
        from paper_2602_01410_amd import snip
        case = s["case"]
        kind, t, c, v = case["kind"], case["tokens"], case["cols"], case["vocab"]
        if kind == "embed_grad":
            n = snip.embed_workspace_bytes(t, c, v)
        else:
            n = (snip.vocab_loss_backward_workspace_bytes if kind.endswith("_grad") else snip.vocab_loss_workspace_bytes)(t, c, v, case.get("k", 1))
        s["scratch"] = torch.empty(n, dtype=torch.uint8, device="cuda")
    return s["scratch"]


def _own(s):
    from paper_2602_01410_amd import snip

    case = s["case"]
    kind = case["kind"]
    if kind == "embed":
        snip.snip_embed(s["w"], s["ids"], scale=case["scale"], out=s["y"])
        return s["y"]
    if kind == "embed_grad":
        snip.snip_embed_backward(s["dy"], s["ids"], case["vocab"], scale=case["scale"], dw=s["dw"], accumulate=case["add"], workspace=_scratch(s))
        return s["dw"]
    if kind == "ce":
        snip.snip_cross_entropy(s["x"], s["w"], s["targets"], loss=s["loss"], lse=s["lse"], workspace=_scratch(s))
    elif kind == "distill":
        snip.snip_distill(s["x"], s["w"], s["indices"], s["teacher"], temperature=case["tau"], loss=s["loss"], lse=s["lse"], workspace=_scratch(s))
    elif kind == "ce_grad":
        snip.snip_cross_entropy_backward(s["x"], s["w"], s["targets"], s["lse"], dloss=s["dloss"], dx=s["dx"], dw=s["dw"], workspace=_scratch(s))
    else:
        snip.snip_distill_backward(s["x"], s["w"], s["indices"], s["teacher"], s["lse"], temperature=case["tau"], dloss=s["dloss"], dx=s["dx"], dw=s["dw"],
                                   workspace=_scratch(s))
    return {"dx": s["dx"], "dw": s["dw"]} if kind.endswith("_grad") else {"loss": s["loss"], "lse": s["lse"]}


def run(state):
    if own:
        return _own(state)
    kind = state["case"]["kind"]
    return {"embed": _embed, "embed_grad": _embed_grad}.get(kind, _loss_grad if kind.endswith("_grad") else _loss)(state)


# ---- in 64 bits -----------------------------------------------------------------------------------------------------------


def _wanted(s, rows):
    """Probabilities that the entries of these tokens should have, one list of (entry, probability) columns: an entry outside the vocabulary has none."""
    case = s["case"]
    v = case["vocab"]
    if case["kind"].startswith("ce"):
        at = s["targets"][rows].long().unsqueeze(1)
        valid = at.ge(0) & at.lt(v)
        return at * valid, valid.double()
    at = s["indices"][rows].long()
    valid = at.ge(0) & at.lt(v)
    u = s["teacher"][rows].double().div(case["tau"]).masked_fill(~valid, -math.inf)
    return at * valid, torch.softmax(u, 1).nan_to_num(0.0) * valid


def exact(case, seed):
    s = prepare(case, seed)
    kind, t, v = case["kind"], case["tokens"], case["vocab"]
    if kind == "embed":
        got = torch.zeros(t, case["cols"], dtype=torch.float64, device="cuda")
        known = (s["ids"] >= 0).nonzero()[:, 0]
        got[known] = s["w"].index_select(0, s["ids"][known].long()).double() * case["scale"]
        return got
    if kind == "embed_grad":
        got = s["dw"].double() / case["scale"] if case["add"] else torch.zeros(v, case["cols"], dtype=torch.float64, device="cuda")
        known = (s["ids"] >= 0).nonzero()[:, 0]
        got.index_put_((s["ids"][known].long(),), s["dy"][known].double(), accumulate=True)
        return got * case["scale"]
    tau = case.get("tau", 1.0)
    w = s["w"].double()
    loss, lse = torch.zeros(t, dtype=torch.float64, device="cuda"), torch.zeros(t, dtype=torch.float64, device="cuda")
    grads = kind.endswith("_grad")
    if grads:
        dx, dw = torch.zeros(t, case["cols"], dtype=torch.float64, device="cuda"), torch.zeros_like(w)
    for first in range(0, t, 1024):
        rows = slice(first, min(t, first + 1024))
        x = s["x"][rows].double()
        logits = torch.mm(x, w.t()).div_(tau)
        at, want = _wanted(s, rows)
        if grads:
            # from the statistic that the call is given
            p = logits.sub_(s["lse"][rows].double().unsqueeze(1)).exp_()
            p.mul_(want.sum(1).gt(0).double().unsqueeze(1))
            p.scatter_add_(1, at, want.neg())
            p.mul_((s["dloss"][rows].double() * tau).unsqueeze(1))
            dx[rows] = torch.mm(p, w)
            dw.addmm_(p.t(), x)
        else:
            lse[rows] = torch.logsumexp(logits, 1)
            log_p = logits.gather(1, at) - lse[rows].unsqueeze(1)
            loss[rows] = torch.xlogy(want, want).sub_(want * log_p).sum(1).mul_(tau * tau)
    return {"dx": dx, "dw": dw} if grads else {"loss": loss, "lse": lse}
