"""The operators around the quantized linear layer, as a program calls them: what makes its input (RMS norm with the
residual's addition, quantized outputs, and the norm's gradient), what takes its weight gradient (an AdamW step over
many tensors) and what answers with its weights (few tokens against FP4 / FP8 weights).

`run` computes them with elementary torch operations in 32 bits, or, where `own` is set, with the calls of
`paper_2602_01410_amd.snip`.  What has 8 bits is returned as torch's 8-bit floating types; FP4 values, which torch has no type
to compute with, as the E5M2 numbers that they are.
"""
from __future__ import annotations

import math

import torch

own = False

E4M3, E8M0, E5M2 = torch.float8_e4m3fn, torch.float8_e8m0fnu, torch.float8_e5m2
BLOCK = 128             # elements that share the scale of an 8-bit optimizer state
ROOT_MAX = 1.9375       # largest number of the unsigned 8-bit format of sqrt(v)
LR, BETA1, BETA2, EPS, STEP = 1e-4, 0.9, 0.95, 1e-8, 100

# The linears of a block with their norms' gains, by the shapes of this repository's configurations.
BLOCK_1B = "2048x2048,2048x2048,2048x2048,2048x2048,8192x2048,8192x2048,2048x8192,2048,2048"
BLOCK_7B = "4096x4096,4096x4096,4096x4096,4096x4096,11008x4096,11008x4096,4096x11008,4096,4096"


def listed():
    return [
        # generation, one token: the norm between two sub-blocks of a 7B-shaped model; launches are all there is
        {"name": "norm_1x4096_y", "kind": "norm", "rows": 1, "cols": 4096, "residual": True, "gain": "bf16", "y": True, "row": 0, "col": 0, "pad": 0},
        # a short ragged batch in FP4 along rows only, as an evaluation needs it; fp32 gains, padded rows
        {"name": "norm_250x2080_row4", "kind": "norm", "rows": 250, "cols": 2080, "residual": False, "gain": "fp32", "y": False, "row": 4, "col": 0, "pad": 24},
        # training steps: both orientations in FP8, what the forward and the weight-gradient GEMM read: 1B- and 7B-shaped
        {"name": "norm_4096x2048_both8", "kind": "norm", "rows": 4096, "cols": 2048, "residual": True, "gain": "bf16", "y": False, "row": 8, "col": 8, "pad": 0},
        {"name": "norm_16384x4096_both8", "kind": "norm", "rows": 16384, "cols": 4096, "residual": True, "gain": "bf16", "y": False, "row": 8, "col": 8, "pad": 0},
        # gradients: the first norm of a model (nothing flows past it) over an odd batch; a 70B-shaped one with the residual's gradient
        {"name": "norm_grad_1501x2056", "kind": "norm_grad", "rows": 1501, "cols": 2056, "residual": False, "gain": "fp32", "pad": 0},
        {"name": "norm_grad_8192x8192", "kind": "norm_grad", "rows": 8192, "cols": 8192, "residual": True, "gain": "bf16", "pad": 0},
        # optimizer: a single small linear with its norm; a 7B-shaped block, bf16 gradients as the wgrad calls write them
        {"name": "adamw_32_small", "kind": "adamw", "sizes": "512x512,512", "bits": 32, "grad": "fp32", "copy": True},
        {"name": "adamw_32_7b_block", "kind": "adamw", "sizes": BLOCK_7B, "bits": 32, "grad": "bf16", "copy": True},
        # a 1B-shaped block with 8-bit states
        {"name": "adamw_8_1b_block", "kind": "adamw", "sizes": BLOCK_1B, "bits": 8, "grad": "bf16", "copy": True},
        # generation: one token through q, k and v of a 7B-shaped block, which share their input; nine sequences through an odd
        # width in the mixed formats of a plan; 48 sequences through a 70B-shaped gate and up
        {"name": "gemv_1_qkv_4096_fp4", "kind": "gemv", "tokens": 1, "widths": "4096,4096,4096", "k": 4096, "fmts": "444", "out": "bf16"},
        {"name": "gemv_9_1003_2080_84", "kind": "gemv", "tokens": 9, "widths": "1003,1003", "k": 2080, "fmts": "84", "out": "fp32"},
        {"name": "gemv_48_gate_up_70b_fp4", "kind": "gemv", "tokens": 48, "widths": "28672,28672", "k": 8192, "fmts": "44", "out": "bf16"},
    ]


def _log_int(rng, lo, hi):
    return max(lo, min(hi, round(math.exp(rng.uniform(math.log(lo), math.log(hi + 0.5))))))


def _to(v, step):
    return max(step, (v + step // 2) // step * step)


def draw(rng):
    kind = rng.choice(("norm", "norm", "norm_grad", "adamw", "gemv", "gemv"))
    if kind in ("norm", "norm_grad"):
        cols = _log_int(rng, 64, 16384)
        rows = _log_int(rng, 1, min(16384, (1 << 25) // cols if kind == "norm" else (1 << 26) // cols))
        c = {"kind": kind, "rows": rows, "cols": cols, "residual": rng.random() < 0.7, "gain": rng.choice(("bf16", "bf16", "fp32")),
             "pad": rng.choice((0, 0, 8, 40))}
        if kind == "norm_grad":
            return c
        form = rng.choice(("y", "row", "both", "both"))
        if form != "y":
            c["cols"] = _to(cols, 32)
        if form == "both":
            c["rows"] = _to(rows, 32)
        fmt = lambda: 4 if rng.random() < 0.15 else 8  # noqa: E731
        return c | {"y": form == "y" or rng.random() < 0.2, "row": fmt() if form != "y" else 0, "col": fmt() if form == "both" else 0}
    if kind == "adamw":
        sizes, left = [], 1 << 26
        for _ in range(rng.randint(1, 24)):
            r, k = _log_int(rng, 16, 8192), _log_int(rng, 16, 8192)
            if r * k <= left:
                sizes.append("%dx%d" % (r, k))
                left -= r * k
            sizes.append(str(_log_int(rng, 1, 8192)))
        return {"kind": kind, "sizes": ",".join(sizes), "bits": rng.choice((32, 8)), "grad": rng.choice(("bf16", "bf16", "fp32")), "copy": rng.random() < 0.8}
    k, n = _to(_log_int(rng, 256, 16384), 32), rng.randint(1, 3)
    widths = [_log_int(rng, 64, min(28672, (1 << 28) // (k * n))) for _ in range(n)]
    return {"kind": kind, "tokens": _log_int(rng, 1, 48), "widths": ",".join(map(str, widths)), "k": k,
            "fmts": "".join("4" if rng.random() < 0.7 else "8" for _ in widths), "out": rng.choice(("bf16", "bf16", "fp32"))}


def _shapes(case):
    return [tuple(int(v) for v in s.split("x")) for s in case["sizes"].split(",")]


def _code_bytes(n, fmt):
    return n * (fmt / 8 + 1 / 32)


def work(case):
    kind = case["kind"]
    if kind == "norm":
        n, gain = case["rows"] * case["cols"], case["cols"] * (4 if case["gain"] == "fp32" else 2)
        out = (2 * n if case["y"] else 0) + sum(_code_bytes(n, case[o]) for o in ("row", "col") if case[o])
        return {"bytes": n * (6 if case["residual"] else 2) + gain + 4 * case["rows"] + out, "flops": 5 * n}
    if kind == "norm_grad":
        n, gain = case["rows"] * case["cols"], case["cols"] * (8 if case["gain"] == "fp32" else 6)
        return {"bytes": n * (8 if case["residual"] else 6) + gain + 4 * case["rows"], "flops": 10 * n}
    if kind == "adamw":
        n = sum(math.prod(s) for s in _shapes(case))
        state = 16 if case["bits"] == 32 else 4 + 16 / BLOCK
        return {"bytes": n * (8 + state + (2 if case["grad"] == "bf16" else 4) + (2 if case["copy"] else 0)), "flops": 15 * n}
    k, m, widths = case["k"], case["tokens"], [int(v) for v in case["widths"].split(",")]
    weights = sum(_code_bytes(w * k, int(f)) for w, f in zip(widths, case["fmts"]))
    return {"bytes": weights + 2 * m * k + (2 if case["out"] == "bf16" else 4) * m * sum(widths), "flops": 2 * m * k * sum(widths)}


# ---- inputs ---------------------------------------------------------------------------------------------------------------


def _rows(gen, rows, cols, pad, std=1.0):
    """A bf16 matrix whose rows are apart by a multiple of 8 elements; one column in a hundred is an outlier column."""
    ld = (cols + 7) // 8 * 8 + pad
    t = torch.randn(rows, ld, generator=gen, device="cuda")
    t *= 1 + 15 * (torch.rand(ld, generator=gen, device="cuda") < 0.01)
    return (t * std).bfloat16()[:, :cols]


def _gain(gen, cols, kind):
    return (1 + 0.1 * torch.randn(cols, generator=gen, device="cuda")).to(torch.float32 if kind == "fp32" else torch.bfloat16)


def _empty_codes(rows, cols, fmt):
    return {"codes": torch.empty(rows, cols * fmt // 8, dtype=torch.uint8, device="cuda"), "rows": rows, "cols": cols, "fmt": fmt,
            "scales": torch.empty(rows, cols // 32, dtype=torch.uint8, device="cuda"),
            # the second copy of the scales that the GEMMs read
            "grouped": torch.empty((cols + 127) // 128, (rows + 255) // 256 * 256, 4, dtype=torch.uint8, device="cuda")}


def _pack4(values):
    """Nibbles of numbers on the E2M1 grid, the first of a pair in the low half."""
    a = values.abs()
    nib = torch.where(a < 2, a * 2, torch.where(a < 4, a + 2, a / 2 + 4)).to(torch.uint8) | (torch.signbit(values).to(torch.uint8) << 3)
    return nib[..., 0::2] | (nib[..., 1::2] << 4)


def prepare(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    kind = case["kind"]
    s = {"case": case}
    if kind in ("norm", "norm_grad"):
        rows, cols, pad = case["rows"], case["cols"], case["pad"]
        s["x"] = _rows(gen, rows, cols, pad)
        s["gain"] = _gain(gen, cols, case["gain"])
        s["dx" if kind == "norm_grad" else "sum"] = torch.empty(rows, s["x"].stride(0), dtype=torch.bfloat16, device="cuda")[:, :cols]
        if rows > 8:
            s["x"][rows // 2] = 0             # a padding token
        if kind == "norm_grad":
            x = s["x"].float()
            s["rstd"] = (x.square().mean(1) + 1e-5).rsqrt()
            s["dy"] = _rows(gen, rows, cols, pad, 1e-4)
            s["dsum"] = _rows(gen, rows, cols, pad, 1e-4) if case["residual"] else None
            s["dgain"] = torch.empty(cols, device="cuda")
            s["scratch"] = torch.empty(1 << 25, dtype=torch.uint8, device="cuda")
            return s
        s["residual"] = _rows(gen, rows, cols, pad, 3.0) if case["residual"] else None
        if case["residual"] and rows > 8:
            s["residual"][rows // 2] = 0
        s["rstd"] = torch.empty(rows, device="cuda")
        s["y"] = torch.empty(rows, cols if cols % 8 == 0 else (cols + 7) // 8 * 8, dtype=torch.bfloat16, device="cuda")[:, :cols] if case["y"] else None
        s["row"] = _empty_codes(rows, cols, case["row"]) if case["row"] else None
        s["col"] = _empty_codes(cols, rows, case["col"]) if case["col"] else None
        return s
    if kind == "adamw":
        # one buffer of each kind holds all tensors, each from a multiple of 128 elements on
        shapes = _shapes(case)
        counts = [math.prod(v) for v in shapes]
        first = [0]
        for n in counts:
            first.append(first[-1] + (n + BLOCK - 1) // BLOCK * BLOCK)
        total, blocks = first[-1], first[-1] // BLOCK
        used = torch.zeros(total, dtype=torch.bool, device="cuda")
        for n, f in zip(counts, first):
            used[f:f + n] = True
        std = 1e-3
        s["grad"] = (torch.randn(total, generator=gen, device="cuda") * (std * used)).to(torch.bfloat16 if case["grad"] == "bf16" else torch.float32)
        s["p"] = torch.randn(total, generator=gen, device="cuda") * (0.02 * used)
        m = torch.randn(total, generator=gen, device="cuda") * (std * math.sqrt((1 - BETA1) / (1 + BETA1)) * used)
        v = std ** 2 * (1 + 0.15 * torch.randn(total, generator=gen, device="cuda")).clamp_(0.2) * used
        if case["bits"] == 32:
            s["m"], s["v"] = m, v
        else:
            s["m"], s["m_scale"] = _moment_codes(m.view(-1, BLOCK))
            s["v"], s["v_scale"] = _root_codes(v.sqrt().view(-1, BLOCK), torch.full((blocks, BLOCK), 0x8000, device="cuda"))
            s["m"], s["v"] = s["m"].view(-1), s["v"].view(-1)
        del m, v
        s["copy"] = s["p"].bfloat16() if case["copy"] else None
        s["grad_scale"] = torch.full((1,), 0.75, device="cuda")
        s["seed"] = seed * 2654435761 % (1 << 64)
        # matrices decay, gains do not
        s["decay"] = [0.1 if len(v) == 2 else 0.0 for v in shapes]
        s["spans"] = list(zip(first, counts))
        # of every group of 128 elements: its decay, its tensor and its place in that tensor
        per = torch.tensor([(b - a) // BLOCK for a, b in zip(first, first[1:])], device="cuda")
        s["of_tensor"] = torch.repeat_interleave(torch.arange(len(counts), device="cuda"), per)
        s["place"] = torch.arange(blocks, device="cuda") - torch.tensor(first[:-1], device="cuda")[s["of_tensor"]] // BLOCK
        s["decays"] = torch.tensor(s["decay"], device="cuda")[s["of_tensor"]]
        return s
    m, k = case["tokens"], case["k"]
    s["x"] = _rows(gen, m, k, 0)
    s["weights"], s["y"] = [], []
    for n, f in zip(case["widths"].split(","), case["fmts"]):
        w = torch.randn(int(n), k, generator=gen, device="cuda") * 0.02
        values, byte = _blocks(w, int(f))
        codes = _pack4(values) if f == "4" else values.to(E4M3).view(torch.uint8)
        s["weights"].append({"codes": codes, "scales": byte, "rows": int(n), "cols": k, "fmt": int(f)})
        pitch = (int(n) + 7) // 8 * 8
        s["y"].append(torch.empty(m, pitch, dtype=torch.bfloat16 if case["out"] == "bf16" else torch.float32, device="cuda")[:, :int(n)])
    return s


# ---- plain forms ----------------------------------------------------------------------------------------------------------


def _blocks(y, fmt):
    """Numbers of the format, before their scale, and scale bytes of the groups of 32 along y's rows."""
    g = y.reshape(y.shape[0], -1, 32)
    bits = g.abs().amax(2).view(torch.int32)
    # the smallest power of two under which the largest fits: its exponent, one more where the mantissa is over the format's largest
    byte = ((bits + (0x1FFFFF if fmt == 8 else 0x3FFFFF)) >> 23) - (8 if fmt == 8 else 2)
    byte = byte.clamp(0, 254)
    v = torch.ldexp(g, (127 - byte).unsqueeze(2))
    if fmt == 8:
        v = v.to(E4M3).float()
    else:
        a = v.abs()
        step = torch.where(a < 2, 0.5, torch.where(a < 4, 1.0, 2.0))
        v = torch.copysign(torch.round(a / step) * step, v)
    return v.view_as(y), byte.to(torch.uint8)


def _quantized(y, fmt):
    values, byte = _blocks(y, fmt)
    if fmt == 8:
        return {"codes": values.to(E4M3), "scales": byte.view(E8M0)}
    return {"values": _scaled4(values, byte)}


def _scaled4(values, byte):
    return torch.ldexp(values.reshape(values.shape[0], -1, 32), byte.int().unsqueeze(2) - 127).view_as(values).to(E5M2)


def _unpack4(codes):
    grid = torch.tensor([0., .5, 1., 1.5, 2., 3., 4., 6., -0., -.5, -1., -1.5, -2., -3., -4., -6.], device=codes.device)
    return grid[torch.stack((codes & 15, codes >> 4), 2).int()].view(codes.shape[0], -1)


def _weights(w):
    v = _unpack4(w["codes"]) if w["fmt"] == 4 else w["codes"].view(E4M3).float()
    return (v.view(w["rows"], -1, 32) * torch.ldexp(torch.ones((), device=v.device), w["scales"].int() - 127).unsqueeze(2)).view(w["rows"], -1)


def _norm(s):
    x = s["x"].float()
    if s["residual"] is not None:
        s["sum"].copy_(x + s["residual"].float())
        x = s["sum"].float()
    rstd = (x.square().mean(1) + 1e-5).rsqrt()
    y = x * rstd[:, None] * s["gain"].float()
    got = {"rstd": rstd}
    if s["residual"] is not None:
        got["sum"] = s["sum"]
    if s["y"] is not None:
        got["y"] = y.bfloat16()
    if s["row"] is not None:
        got["row"] = _quantized(y, s["row"]["fmt"])
    if s["col"] is not None:
        got["col"] = _quantized(y.t().contiguous(), s["col"]["fmt"])
    return got


def _norm_grad(s):
    x, dy, rstd = s["x"].float(), s["dy"].float(), s["rstd"][:, None]
    g = dy * s["gain"].float()
    dx = rstd * (g - x * (rstd * rstd * (g * x).mean(1, keepdim=True)))
    if s["dsum"] is not None:
        dx = dx + s["dsum"].float()
    return {"dx": dx.bfloat16(), "dgain": (dy * (x * rstd)).sum(0)}


def _scale(largest, most):
    """Scales that take the largest of a group to `most`, and their reciprocals; none for a group below the normal numbers."""
    scale = largest * (1 / most)
    scale = torch.where(scale < 2.0 ** -126, 0.0, scale)
    return scale, torch.where(scale == 0, 0.0, 1 / scale)[:, None]


def _moment_codes(m):
    """E4M3 numbers and the scale of each row of 128."""
    scale, inverse = _scale(m.abs().amax(1), 448)
    return (m * inverse).to(E4M3), scale


def _root_codes(r, rnd):
    """sqrt(v) as unsigned 8-bit numbers with 4 exponent and 4 mantissa bits (those of a half below 2, without its 6 last bits),
    rounded up where the dropped bits and the 16 random ones carry; what is not zero stays so."""
    scale, inverse = _scale(r.amax(1), ROOT_MAX)
    t = r * inverse
    c = ((t * 2.0 ** -112).view(torch.int32) + (rnd.int() << 3)) >> 19
    return torch.where(t > 0, c.clamp(1, 255), 0).to(torch.uint8), scale


def _root_values(c):
    return torch.bitwise_left_shift(c, torch.full((1,), 6, dtype=torch.int16, device=c.device)).view(torch.float16)


def _threefry(c0, c1, seed):
    """Threefry-2x32 with 20 rounds (Salmon et al., SC'11) on 32-bit words held in 64."""
    low = 0xFFFFFFFF
    keys = [seed & low, seed >> 32]
    keys.append(0x1BD11BDA ^ keys[0] ^ keys[1])
    x0, x1 = (c0 + keys[0]) & low, (c1 + keys[1]) & low
    for r in range(20):
        x0 = (x0 + x1) & low
        k = (13, 15, 26, 6, 17, 29, 16, 24)[r % 8]
        x1 = (((x1 << k) | (x1 >> (32 - k))) & low) ^ x0
        if r % 4 == 3:
            i = r // 4 + 1
            x0, x1 = (x0 + keys[i % 3]) & low, (x1 + keys[(i + 1) % 3] + i) & low
    return x0, x1


def _random16(s):
    """16 random bits for every element: a call of the generator gives four elements theirs; its counter is the place in the tensor over
    four and the tensor's number."""
    quads = s["place"][:, None] * (BLOCK // 4) + torch.arange(BLOCK // 4, device="cuda")
    o0, o1 = _threefry(quads, s["of_tensor"][:, None].expand_as(quads), s["seed"])
    return torch.stack((o0 & 0xFFFF, o0 >> 16, o1 & 0xFFFF, o1 >> 16), 2).view(-1, BLOCK)


def _adamw(s):
    small = s["case"]["bits"] == 8
    grad = s["grad"].float() * s["grad_scale"]
    if small:
        m = (s["m"].view(E4M3).float().view(-1, BLOCK) * s["m_scale"][:, None]).view(-1)
        v = (_root_values(s["v"]).float().view(-1, BLOCK) * s["v_scale"][:, None]).view(-1).square()
    else:
        m, v = s["m"], s["v"]
    m = BETA1 * m + (1 - BETA1) * grad
    v = BETA2 * v + (1 - BETA2) * grad.square()
    step = (m / (1 - BETA1 ** STEP)) / ((v / (1 - BETA2 ** STEP)).sqrt() + EPS)
    p = s["p"].view(-1, BLOCK)
    s["p"].copy_((p * (1 - LR * s["decays"])[:, None] - LR * step.view(-1, BLOCK)).view(-1))
    got = {"p": s["p"]}
    if small:
        mc, ms = _moment_codes(m.view(-1, BLOCK))
        vc, vs = _root_codes(v.sqrt().view(-1, BLOCK), _random16(s))
        s["m"].copy_(mc.view(-1)), s["v"].copy_(vc.view(-1)), s["m_scale"].copy_(ms), s["v_scale"].copy_(vs)
    else:
        s["m"].copy_(m), s["v"].copy_(v)
    if s["copy"] is not None:
        s["copy"].copy_(s["p"])
    return got | _states(s)


def _states(s):
    got = {"m": s["m"], "v": s["v"]}
    if s["copy"] is not None:
        got["copy"] = s["copy"]
    if s["case"]["bits"] == 8:
        got |= {"v": _root_values(s["v"]), "m_scale": s["m_scale"], "v_scale": s["v_scale"]}
    return got


def _gemv(s):
    x = s["x"].float()
    return [(x @ _weights(w).t()).to(y.dtype) for w, y in zip(s["weights"], s["y"])]


# ---- the framework's calls ------------------------------------------------------------------------------------------------


def _own(s):
    from paper_2602_01410_amd import snip

    def q(d, grouped=True):
        return snip.QTensor(d["codes"], d["scales"], d["rows"], d["cols"], snip.FP8 if d["fmt"] == 8 else snip.FP4, d["grouped"] if grouped else None)

    kind = s["case"]["kind"]
    if kind == "norm":
        outs = {o: q(s[o]) for o in ("row", "col") if s[o] is not None}
        snip.snip_rms_norm(s["x"], s["gain"], 1e-5, residual=s["residual"], sum=s["sum"] if s["residual"] is not None else None, rstd=s["rstd"],
                           y=s["y"], out_row=outs.get("row"), out_col=outs.get("col"))
        got = {"rstd": s["rstd"]}
        if s["residual"] is not None:
            got["sum"] = s["sum"]
        if s["y"] is not None:
            got["y"] = s["y"]
        for o, t in outs.items():
            got[o] = {"codes": t.codes.view(E4M3), "scales": t.scales.view(E8M0)} if t.fmt == snip.FP8 else {"values": _scaled4(_unpack4(t.codes), t.scales)}
        return got
    if kind == "norm_grad":
        snip.snip_rms_norm_backward(s["dy"], s["x"], s["gain"], s["rstd"], dsum=s["dsum"], dx=s["dx"], dweight=s["dgain"], workspace=s["scratch"])
        return {"dx": s["dx"], "dgain": s["dgain"]}
    if kind == "adamw":
        small = s["case"]["bits"] == 8
        tensors = []
        for (f, n), decay in zip(s["spans"], s["decay"]):
            b = slice(f // BLOCK, f // BLOCK + (n + BLOCK - 1) // BLOCK)
            tensors.append(snip.AdamwTensor(s["p"][f:f + n], s["grad"][f:f + n], s["m"].view(torch.uint8)[f:f + n] if small else s["m"][f:f + n], s["v"][f:f + n],
                                            copy=s["copy"][f:f + n] if s["copy"] is not None else None, weight_decay=decay,
                                            m_scale=s["m_scale"][b] if small else None, v_scale=s["v_scale"][b] if small else None))
        snip.snip_adamw_step(tensors, LR, BETA1, BETA2, EPS, STEP, grad_scale=s["grad_scale"], seed=s["seed"])
        return {"p": s["p"]} | _states(s)
    snip.snip_gemv(s["x"], [q(w, False) for w in s["weights"]], s["y"])
    return s["y"]


def run(state):
    if own:
        return _own(state)
    return {"norm": _norm, "norm_grad": _norm_grad, "adamw": _adamw, "gemv": _gemv}[state["case"]["kind"]](state)


# ---- in 64 bits -----------------------------------------------------------------------------------------------------------


def exact(case, seed):
    """Codes have no value here: an element next to the middle between two of them may go either way."""
    s = prepare(case, seed)
    kind = case["kind"]
    if kind == "norm":
        h = s["x"].double()
        got = {"row": None, "col": None}
        if case["residual"]:
            # what is normed is the sum as it is stored; it has no bits that 32 would lose where it matters to bf16
            got["sum"] = h + s["residual"].double()
            h = got["sum"].bfloat16().double()
        ms = torch.einsum("ij,ij->i", h, h) / case["cols"]
        got["rstd"] = 1 / torch.sqrt(ms + 1e-5)
        if case["y"]:
            got["y"] = torch.einsum("ij,i,j->ij", h, got["rstd"], s["gain"].double())
        return got
    if kind == "norm_grad":
        x, dy, rstd = s["x"].double(), s["dy"].double(), s["rstd"].double()
        xhat = torch.einsum("ij,i->ij", x, rstd)
        g = dy * s["gain"].double()
        along = torch.einsum("ij,ij->i", g, xhat) / case["cols"]
        dx = torch.einsum("ij,i->ij", g - torch.einsum("ij,i->ij", xhat, along), rstd)
        if s["dsum"] is not None:
            dx += s["dsum"].double()
        return {"dx": dx, "dgain": torch.einsum("ij,ij->j", dy, xhat)}
    if kind == "adamw":
        small = case["bits"] == 8
        g = s["grad"].double() * 0.75
        if small:
            per = torch.arange(g.numel(), device="cuda") // BLOCK
            m = s["m"].view(E4M3).double() * s["m_scale"].double()[per]
            c = s["v"].double()
            root = torch.where(c >= 16, torch.exp2(torch.floor(c / 16) - 15) * (1 + c.remainder(16) / 16), c * 2.0 ** -18) * s["v_scale"].double()[per]
            v = root * root
        else:
            m, v = s["m"].double(), s["v"].double()
        m.lerp_(g, 1 - BETA1)
        v.lerp_(g.mul_(g), 1 - BETA2)
        del g
        update = v.div(1 - BETA2 ** STEP).sqrt_().add_(EPS).reciprocal_().mul_(m).mul_(LR / (1 - BETA1 ** STEP))
        p = s["p"].double()
        p *= 1 - LR * torch.repeat_interleave(s["decays"].double(), BLOCK)
        p -= update
        got = {"p": p, "m": None, "v": None} if small else {"p": p, "m": m, "v": v}
        if case["copy"]:
            got["copy"] = p
        if small:
            got |= {"m_scale": m.view(-1, BLOCK).abs().amax(1) / 448, "v_scale": v.sqrt().view(-1, BLOCK).amax(1) / ROOT_MAX}
        return got
    x, ys = s["x"].double(), []
    for w in s["weights"]:
        if w["fmt"] == 8:
            v = w["codes"].view(E4M3).double()
        else:
            nib = torch.stack((w["codes"] & 15, w["codes"] >> 4), 2).view(w["rows"], -1).double()
            mag = nib.remainder(8)
            e = torch.floor(mag / 2)
            v = torch.where(e > 0, torch.exp2(e - 1) * (1 + mag.remainder(2) / 2), mag / 2) * (1 - 2 * torch.floor(nib / 8))
            del nib, mag, e
        v *= torch.repeat_interleave(torch.exp2(w["scales"].double() - 127), 32, 1)
        ys.append(x @ v.t())
    return ys
