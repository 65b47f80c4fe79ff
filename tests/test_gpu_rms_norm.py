"""RMS norm with residual and quantized outputs, and its gradient, against 64-bit arithmetic.

What the kernels round in fp32 moves y by at most DELTA, relatively: a row's squares are added one after the other at most
64 times in a lane (cols <= 2^18 here), then over 64 lanes and 16 waves, half of which reaches rstd; mean, root, reciprocal and the
products add 2^-24 each: (64 + 6 + 16) / 2 * 2^-24 + 6 * 2^-24 < 3e-6.  A rounded output then lies between the roundings of
y (1 - DELTA) and y (1 + DELTA)."""
import numpy as np
import pytest
import torch

from paper_2602_01410_amd import snip

pytestmark = pytest.mark.gpu
DELTA = 3e-6
CANARY = 0x7A7A


def bf16(t):
    return t.to(torch.bfloat16)


def rows_of(rng, rows, cols, pad=0, std=1.0):
    """bf16 [rows, cols] on the GPU with a pitch of its own, and its values in 64 bits."""
    ld = (cols + 7) // 8 * 8 + pad
    buf = torch.full((rows, ld), CANARY, dtype=torch.int16, device="cuda").view(torch.bfloat16)
    v = torch.from_numpy((rng.standard_normal((rows, cols)) * std * np.where(rng.random(cols) < 0.02, 20, 1)).astype(np.float32)).to(torch.bfloat16)
    buf[:, :cols] = v.cuda()
    return buf[:, :cols]


def empty_rows(rows, cols, pad=0):
    return torch.full((rows, (cols + 7) // 8 * 8 + pad), CANARY, dtype=torch.int16, device="cuda").view(torch.bfloat16)[:, :cols]


def untouched(view):
    """Whether nothing behind the columns of a view made above was written."""
    rows, cols, ld = view.shape[0], view.shape[1], view.stride(0)
    whole = torch.as_strided(view, (rows, ld), (ld, 1)).view(torch.int16)
    return bool((whole[:, cols:] == CANARY).all())


def f64(t):
    return t.float().cpu().numpy().astype(np.float64)


def gain_of(rng, cols, fp32):
    return torch.from_numpy((1 + 0.2 * rng.standard_normal(cols)).astype(np.float32)).to(torch.float32 if fp32 else torch.bfloat16).cuda()


EMAX, MOST = {8: 8, 4: 2}, {8: 448.0, 4: 6.0}


def scale_exponents(amax, bits, rule):
    """Of every block, by the definition: the smallest power of two under which the largest element fits, or the floor rule's."""
    m, e = np.frexp(np.where(amax > 0, amax, 1.0))          # amax = 2 m 2^(e-1)
    n = e - 1
    out = n - EMAX[bits]
    if rule == snip.NO_OVERFLOW:
        out = out + (2 * m > MOST[bits] / 2.0 ** EMAX[bits])
    return np.where(amax > 0, np.clip(out, -127, 127), -127)


def round_code(v, bits):
    """|v| to the nearest number of the format, ties to even, saturating."""
    a = np.minimum(np.abs(v), MOST[bits])
    low, mant = (-6, 3) if bits == 8 else (0, 1)
    e = np.maximum(np.floor(np.log2(np.where(a > 0, a, 1.0))), low)
    step = 2.0 ** (e - mant)
    return np.minimum(np.rint(a / step) * step, MOST[bits])


def decode(q):
    """Code numbers (without scales) and scale bytes in numpy."""
    c = q.codes.cpu()
    if q.fmt == snip.FP8:
        v = c.view(torch.float8_e4m3fn).double().numpy()
    else:
        grid = np.array([0, .5, 1, 1.5, 2, 3, 4, 6])
        c = c.numpy()
        nib = np.stack((c & 15, c >> 4), 2).reshape(c.shape[0], -1)
        v = np.where(nib & 8, -grid[nib & 7], grid[nib & 7])
    return v, q.scales.cpu().numpy().astype(np.int64)


def check_codes(q, y, rule):
    """Codes and scales of q are those of y, up to DELTA; the grouped copy holds the same scales."""
    bits = 8 if q.fmt == snip.FP8 else 4
    v, byte = decode(q)
    blocks = np.abs(y).reshape(y.shape[0], -1, 32)
    lo, hi = (scale_exponents(blocks.max(2) * f, bits, rule) + 127 for f in (1 - DELTA, 1 + DELTA))
    finite = np.isfinite(blocks).all(2)
    assert ((byte >= lo) & (byte <= hi))[finite].all()
    assert (byte[~finite] == 255).all()
    s = np.repeat(2.0 ** (byte - 127.0), 32, 1)
    fin = np.repeat(finite, 32, 1)
    with np.errstate(invalid="ignore"):
        a, b = (round_code(y / s * f, bits) for f in (1 - DELTA, 1 + DELTA))
    assert ((np.abs(v) >= a) & (np.abs(v) <= b))[fin].all()
    assert ((v == 0) | (np.sign(v) == np.sign(y)))[fin].all()
    assert (v[~fin] == 0).all()
    g4 = q.scales_g4.cpu().numpy()
    nb = byte.shape[1]
    for k in range(nb):
        assert (g4[k // 4, :q.rows, k % 4] == byte[:, k]).all()


def between(got, ref):
    """bf16 numbers between the roundings of ref (1 -+ DELTA)."""
    r = torch.from_numpy(np.abs(ref))
    lo, hi = (bf16((r * f).float()).double().numpy() for f in (1 - DELTA, 1 + DELTA))
    a = np.abs(got)
    assert ((a >= lo) & (a <= hi)).all()
    assert ((got == 0) | (np.sign(got) == np.sign(ref))).all()


def reference(h, w, eps):
    with np.errstate(invalid="ignore", over="ignore", divide="ignore"):
        rstd = 1 / np.sqrt((h * h).mean(1) + eps)
        return rstd, h * rstd[:, None] * w


SHAPES = [(1, 8), (1, 32), (3, 1), (5, 13), (4, 129), (33, 512), (2, 520), (6, 1024), (9, 2048), (7, 2056), (1, 4096), (5, 4104), (3, 8192),
          (3, 8200), (2, 8191), (2, 16384), (2, 16391), (2, 32768), (1, 32776), (2, 40001)]


@pytest.mark.parametrize("residual", [False, True])
@pytest.mark.parametrize("rows,cols", SHAPES)
def test_y_sum_rstd(rows, cols, residual):
    rng = np.random.default_rng(rows * 100003 + cols + residual)
    x, w = rows_of(rng, rows, cols, 8), gain_of(rng, cols, fp32=residual)
    r = rows_of(rng, rows, cols, 16, 3.0) if residual else None
    sum_ = empty_rows(rows, cols, 24) if residual else None
    y = empty_rows(rows, cols, 8)
    got = snip.snip_rms_norm(x, w, 1e-5, residual=r, sum=sum_, y=y)
    assert got.y is y and got.sum is sum_
    h = f64(x)
    if residual:
        h = f64(sum_)
        assert torch.equal(sum_, bf16(x.float() + r.float()))
        assert untouched(sum_)
    rstd, ref = reference(h, f64(w), 1e-5)
    assert np.abs(f64(got.rstd) / rstd - 1).max() <= DELTA
    between(f64(y), ref)
    assert untouched(y) and untouched(x)


@pytest.mark.parametrize("rule", [snip.NO_OVERFLOW, snip.OCP_FLOOR])
@pytest.mark.parametrize("fr,fc", [(snip.FP8, None), (snip.FP4, None), (None, snip.FP8), (None, snip.FP4), (snip.FP8, snip.FP4), (snip.FP4, snip.FP8), (snip.FP8, snip.FP8)])
@pytest.mark.parametrize("rows,cols", [(32, 32), (64, 96), (160, 544), (96, 2048), (256, 160), (288, 4096), (32, 8224)])
def test_codes(rows, cols, fr, fc, rule):
    rng = np.random.default_rng(rows + cols)
    residual = (rows // 32) % 2 == 0
    x, w = rows_of(rng, rows, cols, 8), gain_of(rng, cols, fp32=not residual)
    r = rows_of(rng, rows, cols, 0, 2.0) if residual else None
    got = snip.snip_rms_norm(x, w, 1e-6, residual=r, fmt_row=fr, fmt_col=fc, rule=rule)
    assert got.y is None
    _, ref = reference(f64(got.sum if residual else x), f64(w), 1e-6)
    if fr is not None:
        check_codes(got.row, ref, rule)
    if fc is not None:
        check_codes(got.col, np.ascontiguousarray(ref.T), rule)


@pytest.mark.parametrize("rows,cols", [(544, 544), (544, 1024), (512, 1024), (544, 2080), (544, 4096), (513, 4104), (520, 8192), (257, 1033), (257, 2049), (256, 1033), (100, 1033)])
def test_many_rows(rows, cols):
    """A row's waves depend on the number of rows too."""
    rng = np.random.default_rng(rows * 7 + cols)
    x, r, w = rows_of(rng, rows, cols), rows_of(rng, rows, cols), gain_of(rng, cols, False)
    out = snip.snip_rms_norm(x, w, 1e-5, residual=r, y=empty_rows(rows, cols), fmt_row=snip.FP8 if cols % 32 == 0 else None,
                             fmt_col=snip.FP4 if rows % 32 == 0 and cols % 2 == 0 else None)
    h = f64(out.sum)
    assert (h == f64(bf16(x.float() + r.float()))).all()
    rstd, y = reference(h, f64(w), 1e-5)
    assert (np.abs(f64(out.rstd) / rstd - 1) <= DELTA).all()
    between(f64(out.y), y)
    if out.row is not None:
        check_codes(out.row, y, snip.NO_OVERFLOW)
    if out.col is not None:
        check_codes(out.col, y.T, snip.NO_OVERFLOW)


@pytest.mark.parametrize("rows", [1, 3, 50])
def test_row_codes_of_any_number_of_rows(rows):
    rng = np.random.default_rng(rows)
    x, w = rows_of(rng, rows, 4128), gain_of(rng, 4128, False)
    y = empty_rows(rows, 4128)
    got = snip.snip_rms_norm(x, w, 1e-5, y=y, fmt_row=snip.FP8)
    _, ref = reference(f64(x), f64(w), 1e-5)
    check_codes(got.row, ref, snip.NO_OVERFLOW)
    between(f64(y), ref)


def test_columns_without_blocks_along_rows():
    """Columns need not be a multiple of 32 where only they are blocked."""
    rng = np.random.default_rng(4)
    x, w = rows_of(rng, 64, 134), gain_of(rng, 134, True)
    got = snip.snip_rms_norm(x, w, 1e-5, fmt_col=snip.FP4)
    check_codes(got.col, np.ascontiguousarray(reference(f64(x), f64(w), 1e-5)[1].T), snip.NO_OVERFLOW)


def test_empty_and_non_finite_rows():
    rng = np.random.default_rng(5)
    x, w = rows_of(rng, 64, 160), gain_of(rng, 160, False)
    x[3] = 0                                    # a padding token
    x[7, 5] = float("inf")
    x[40, 100] = float("nan")
    x[41, 3] = -3.3e38                          # its square is no fp32 number: the norm is infinite, y zero
    got = snip.snip_rms_norm(x, w, 1e-5, y=empty_rows(64, 160), fmt_row=snip.FP8, fmt_col=snip.FP8)
    rstd, ref = reference(f64(x), f64(w), 1e-5)
    y = f64(got.y)
    assert (y[3] == 0).all() and np.isclose(float(got.rstd[3]), 1e-5 ** -0.5, rtol=1e-6)
    assert np.isnan(y[7, 5]) and (np.delete(y[7], 5) == 0).all()          # rstd is 0: 0 * inf
    assert np.isnan(y[40]).all() and (y[41] == 0).all()
    v, byte = decode(got.row)
    assert (byte[3] == 0).all() and (v[3] == 0).all()
    assert byte[7, 0] == 255 and (byte[7, 1:] == 0).all() and (byte[40] == 255).all() and (v[40] == 0).all()
    cv, cb = decode(got.col)
    assert (cb[:, 1] == 255).all() and (cv[:, 32:] == 0).all()            # rows 32 to 63 hold row 40
    assert cb[5, 0] == 255 and (np.delete(cb[:, 0], 5) != 255).all()
    ref[[7, 41]] = 0
    keep = [i for i in range(160) if i != 5]
    cols = type(got.col)(got.col.codes[keep][:, :32], got.col.scales[keep][:, :1], 159, 32, snip.FP8, got.col.scales_g4[:, keep])
    check_codes(cols, np.ascontiguousarray(ref.T[keep][:, :32]), snip.NO_OVERFLOW)


@pytest.mark.parametrize("which", ["x", "residual"])
@pytest.mark.parametrize("cols", [96, 4096, 16384, 8191])
def test_sum_in_place(which, cols):
    rng = np.random.default_rng(cols)
    x, r, w = rows_of(rng, 32, cols), rows_of(rng, 32, cols), gain_of(rng, cols, False)
    kw = {"fmt_row": snip.FP8, "fmt_col": snip.FP8} if cols % 32 == 0 else {"y": empty_rows(32, cols)}
    a = snip.snip_rms_norm(x, w, 1e-5, residual=r, **kw)
    b = snip.snip_rms_norm(x, w, 1e-5, residual=r, sum=x if which == "x" else r, **kw)
    assert torch.equal(a.sum, x if which == "x" else r) and torch.equal(a.rstd, b.rstd)
    if cols % 32 == 0:
        assert torch.equal(a.row.codes, b.row.codes) and torch.equal(a.col.codes, b.col.codes) and torch.equal(a.col.scales, b.col.scales)


def grad_reference(dy, h, w, rstd, dsum):
    g = dy * w
    mean = (g * h).mean(1, keepdims=True)
    r = rstd[:, None]
    dx = r * (g - h * r * r * mean)
    parts = r * (np.abs(g) + np.abs(h) * r * r * np.abs(g * h).mean(1, keepdims=True))
    if dsum is not None:
        dx, parts = dx + dsum, parts + np.abs(dsum)
    return dx, parts, (dy * h * r).sum(0), (np.abs(dy * h * r)).sum(0)


def near(got, ref, parts):
    lo, hi = (bf16(torch.from_numpy(ref + e).float()).double().numpy() for e in (-2 * DELTA * parts, 2 * DELTA * parts))
    assert ((got >= lo) & (got <= hi)).all()


@pytest.mark.parametrize("dsum", [False, True])
@pytest.mark.parametrize("rows,cols", SHAPES + [(1200, 64), (2100, 136), (700, 4096), (300, 10000), (530, 21)])
def test_gradient(rows, cols, dsum):
    """dx: between the bf16 roundings of what fp32 may make of its parts (DELTA, and as much again for the second sum).  dweight: at
    most rows + 40 additions and three products per term."""
    rng = np.random.default_rng(rows * 7 + cols)
    h, w = rows_of(rng, rows, cols, 8), gain_of(rng, cols, fp32=dsum)
    dy = rows_of(rng, rows, cols, 0, 1e-3)
    ds = rows_of(rng, rows, cols, 16, 1e-3) if dsum else None
    if rows > 2:
        h[1] = 0
    rstd = torch.from_numpy(reference(f64(h), f64(w), 1e-5)[0].astype(np.float32)).cuda()
    dx = empty_rows(rows, cols, 8)
    _, dw = snip.snip_rms_norm_backward(dy, h, w, rstd, dsum=ds, dx=dx)
    ref, parts, dw_ref, dw_abs = grad_reference(f64(dy), f64(h), f64(w), f64(rstd), f64(ds) if dsum else None)
    near(f64(dx), ref, parts)
    assert (np.abs(f64(dw) - dw_ref) <= (rows + 40) * 2.0 ** -24 * dw_abs + 1e-30).all()
    assert untouched(dx)
    # in place, and without dweight
    was = dx.clone()
    snip.snip_rms_norm_backward(dy, h, w, rstd, dsum=ds, dx=ds if dsum else dy, dweight=dw)
    assert torch.equal(ds if dsum else dy, was)


@pytest.mark.parametrize("rows,cols", [(256, 1024), (257, 520), (301, 1024), (2050, 1016), (1501, 2056), (260, 16384)])
def test_gradient_of_many_rows(rows, cols):
    """A row's waves depend on the number of rows too; bounds as above."""
    test_gradient(rows, cols, True)


def test_gradient_against_differences():
    """Central differences of sum(dy y) in 64 bits; their own error is of the order of step^2."""
    rng = np.random.default_rng(11)
    rows, cols, eps = 4, 96, 1e-5
    x, w, dy = rows_of(rng, rows, cols), gain_of(rng, cols, True), rows_of(rng, rows, cols, 0, 1e-2)
    rstd = snip.snip_rms_norm(x, w, eps).rstd
    dx, dw = snip.snip_rms_norm_backward(dy, x, w, rstd)
    h, wd, d = f64(x), f64(w), f64(dy)
    loss = lambda a, b: (reference(a, b, eps)[1] * d).sum()  # noqa: E731
    dx, dw = f64(dx), f64(dw)
    scale = np.abs(dx).max()
    for _ in range(40):
        i, j = rng.integers(rows), rng.integers(cols)
        e = np.zeros((rows, cols))
        e[i, j] = 1e-4
        diff = (loss(h + e, wd) - loss(h - e, wd)) / 2e-4
        assert abs(diff - dx[i, j]) <= 2.0 ** -8 * abs(diff) + 1e-6 * scale
        e = np.zeros(cols)
        e[j] = 1e-4
        diff = (loss(h, wd + e) - loss(h, wd - e)) / 2e-4
        assert abs(diff - dw[j]) <= 1e-5 * np.abs(dw).max()


def test_no_rows():
    w = torch.ones(64, device="cuda")
    x = torch.empty((0, 64), dtype=torch.bfloat16, device="cuda")
    got = snip.snip_rms_norm(x, w, 1e-5, fmt_row=snip.FP8, fmt_col=snip.FP8)
    assert got.row.rows == 0
    dx, dw = snip.snip_rms_norm_backward(x, x, w, got.rstd)
    assert dx.shape == (0, 64) and (dw == 0).all()


def test_other_stream_and_graph():
    """On a stream of its own, and replayed from a graph with other work in between: the bytes of the eager call."""
    rng = np.random.default_rng(12)
    x, r, w, dy = rows_of(rng, 96, 2048), rows_of(rng, 96, 2048), gain_of(rng, 2048, False), rows_of(rng, 96, 2048)
    a = snip.snip_rms_norm(x, w, 1e-5, residual=r, fmt_row=snip.FP4, fmt_col=snip.FP8)
    dx, dw = snip.snip_rms_norm_backward(dy, a.sum, w, a.rstd, dsum=dy)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    b = snip.snip_rms_norm(x, w, 1e-5, residual=r, fmt_row=snip.FP4, fmt_col=snip.FP8, stream=side)
    dx2, dw2 = snip.snip_rms_norm_backward(dy, b.sum, w, b.rstd, dsum=dy, stream=side)
    side.synchronize()
    ws = torch.empty(snip.rms_norm_workspace_bytes(96, 2048), dtype=torch.uint8, device="cuda")

    def same():
        assert torch.equal(a.row.codes, b.row.codes) and torch.equal(a.col.codes, b.col.codes) and torch.equal(a.col.scales, b.col.scales)
        assert torch.equal(a.row.scales, b.row.scales) and torch.equal(dx, dx2) and torch.equal(dw, dw2) and torch.equal(a.sum, b.sum)

    same()
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        snip.snip_rms_norm(x, w, 1e-5, residual=r, sum=b.sum, rstd=b.rstd, out_row=b.row, out_col=b.col)
        snip.snip_rms_norm_backward(dy, b.sum, w, b.rstd, dsum=dy, dx=dx2, dweight=dw2, workspace=ws)
    for _ in range(3):
        for t in (b.sum, b.rstd, b.row.codes, b.row.scales, b.col.codes, b.col.scales, dx2, dw2, ws):
            t.zero_()
        g.replay()
        torch.cuda.synchronize()
        same()


def test_more_than_2_31_elements():
    rows, cols = 70016, 32768
    gen = torch.Generator(device="cuda").manual_seed(3)
    x = torch.empty((rows, cols), dtype=torch.bfloat16, device="cuda")
    for i in range(0, rows, 8752):
        x[i:i + 8752] = torch.randn((8752, cols), generator=gen, device="cuda")
    w = torch.ones(cols, dtype=torch.bfloat16, device="cuda")
    got = snip.snip_rms_norm(x, w, 1e-5, fmt_row=snip.FP8, fmt_col=snip.FP4)
    for first in (0, 65504, rows - 32):                       # 65536 rows are 2^31 elements
        ref = reference(f64(x[first:first + 32]), f64(w), 1e-5)[1]
        part = lambda q, rs, cs: type(q)(q.codes[rs][:, cs], q.scales[rs][:, :1], 0, 0, q.fmt)  # noqa: E731
        v, byte = decode(type(got.row)(got.row.codes[first:first + 32], got.row.scales[first:first + 32], 32, cols, snip.FP8))
        s = np.repeat(2.0 ** (byte - 127.0), 32, 1)
        assert np.abs(v * s - ref).max() <= 2.0 ** -4 * 1.01 * np.abs(ref).max()
        q = got.col
        v, byte = decode(type(q)(q.codes[:, first // 2:first // 2 + 16].contiguous(), q.scales[:, first // 32:first // 32 + 1].contiguous(), cols, 32, q.fmt))
        amax = np.abs(ref.T).max(1)
        assert (np.abs(v * 2.0 ** (byte - 127.0) - ref.T).max(1) <= amax / 4).all() and (np.abs(v * 2.0 ** (byte - 127.0)).max(1) >= amax / 1.5).all()
    dx, _ = snip.snip_rms_norm_backward(x, x, w, got.rstd)
    for first in (0, 65520, rows - 8):
        h = f64(x[first:first + 8])
        ref, parts, _, _ = grad_reference(h, h, f64(w), f64(got.rstd[first:first + 8]), None)
        near(f64(dx[first:first + 8]), ref, parts)


def test_refusals():
    x = torch.zeros((32, 64), dtype=torch.bfloat16, device="cuda")
    w = torch.ones(64, device="cuda")
    status = lambda f, *a, **k: pytest.raises(snip.SnipError, f, *a, **k).value.status  # noqa: E731
    norm, back = snip.snip_rms_norm, snip.snip_rms_norm_backward
    rstd = torch.ones(32, device="cuda")
    assert status(norm, x, w, -1.0) == 3 and status(norm, x, w, float("nan")) == 3 and status(norm, x, w, 1e-5, rule=2) == 3
    assert status(norm, x, w, 1e-5, sum=x) == 1                                          # a sum of one addend
    assert status(norm, x[:, 4:], w[4:].clone(), 1e-5) == 4                                # rows off 16 bytes
    odd = torch.zeros((32, 66), dtype=torch.bfloat16, device="cuda")[:, :64]
    assert status(norm, odd, w, 1e-5) == 4 and status(back, odd, x, w, rstd) == 4            # pitch
    assert status(norm, x[:, :40], w[:40].clone(), 1e-5, out_row=snip.alloc_qtensor(32, 40, snip.FP8)) == 2
    assert status(norm, x[:24], w, 1e-5, out_col=snip.alloc_qtensor(64, 24, snip.FP8)) == 2
    assert status(norm, x, w, 1e-5, out_row=snip.alloc_qtensor(32, 32, snip.FP8)) == 2       # another matrix's
    assert status(back, x, x, w, rstd, workspace=torch.empty(16, dtype=torch.uint8, device="cuda")) == 5
    for bad in (lambda: norm(x, w[:32], 1e-5), lambda: norm(x, w.half(), 1e-5), lambda: norm(x, w, 1e-5, residual=x[:16]),
                lambda: norm(x, w, 1e-5, rstd=torch.ones(8, device="cuda")), lambda: norm(x.cpu(), w, 1e-5), lambda: back(x, x, w, rstd.double())):
        with pytest.raises(ValueError):
            bad()
