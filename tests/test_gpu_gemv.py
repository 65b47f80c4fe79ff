"""Few tokens against quantized weights.  Products are exact, so that a sum of k of them in fp32, in whatever order, is within k 2^-24 of
the sum of their magnitudes; a bf16 output lies between the roundings of the ends of that interval.  Where every partial sum is a
small multiple of one power of two nothing is rounded, and the outputs are exact."""
import numpy as np
import pytest
import torch

from paper_2602_01410_amd import snip

pytestmark = pytest.mark.gpu
GRID4 = np.array([0, .5, 1, 1.5, 2, 3, 4, 6])
CANARY = 0x7A7A


def weight(rng, n, k, fmt, low=120, high=130):
    """Random codes (none that is not a number) and scale bytes low .. high - 1, and the numbers they stand for."""
    byte = rng.integers(low, high, (n, k // 32)).astype(np.uint8)
    if fmt == snip.FP4:
        nib = rng.integers(0, 16, (n, k)).astype(np.uint8)
        codes = nib[:, 0::2] | nib[:, 1::2] << 4
        v = np.where(nib & 8, -1, 1) * GRID4[nib & 7]
    else:
        c = rng.integers(0, 256, (n, k)).astype(np.uint8)
        c = np.where(c & 0x7F == 0x7F, 0, c).astype(np.uint8)
        codes, v = c, torch.from_numpy(c).view(torch.float8_e4m3fn).double().numpy()
    w = v * np.repeat(2.0 ** (byte - 127.0), 32, 1)
    return snip.QTensor(torch.from_numpy(codes).cuda(), torch.from_numpy(byte).cuda(), n, k, fmt), w


def tokens(rng, m, k, pad=0):
    buf = torch.full((m, k + pad), CANARY, dtype=torch.int16, device="cuda").view(torch.bfloat16)
    x = torch.from_numpy(rng.standard_normal((m, k)).astype(np.float32)).to(torch.bfloat16)
    buf[:, :k] = x.cuda()
    return buf[:, :k], x.double().numpy()


def output(m, n, dtype, pad=0):
    buf = torch.full((m, (n + 7) // 8 * 8 + pad), 31.0, dtype=dtype, device="cuda")
    return buf[:, :n], buf


def check(y, x, w):
    k = x.shape[1]
    ref, room = x @ w.T, k * 2.0 ** -24 * (np.abs(x) @ np.abs(w.T))
    got = y.double().cpu().numpy()
    lo, hi = (torch.from_numpy(ref + e).to(torch.float32).to(y.dtype).double().numpy() for e in (-room, room))
    assert ((got >= lo - 1e-40) & (got <= hi + 1e-40)).all()


@pytest.mark.parametrize("fmt", [snip.FP4, snip.FP8])
@pytest.mark.parametrize("m", [1, 2, 9, 16, 17, 33, 48, 64, 65, 130])
@pytest.mark.parametrize("n,k", [(1, 32), (15, 64), (16, 96), (17, 128), (100, 160), (64, 2080), (1003, 480), (48, 8192)])
def test_against_64_bits(m, n, k, fmt):
    rng = np.random.default_rng(m * n + k)
    x, xd = tokens(rng, m, k, 8 * (m % 3))
    q, w = weight(rng, n, k, fmt)
    for dtype in (torch.bfloat16, torch.float32):
        y, buf = output(m, n, dtype, 8)
        assert snip.snip_gemv(x, [q], [y])[0] is y
        check(y, xd, w)
        assert (buf[:, n:] == 31).all()


@pytest.mark.parametrize("m,n,k", [(15, 33, 4128), (16, 40, 4096), (16, 40, 4128), (13, 9000, 4704), (12, 9000, 5472), (3, 9000, 32), (5, 9000, 11008), (2, 32, 30016), (30, 5000, 1120),
                                   (64, 33000, 544), (40, 18000, 96), (17, 9000, 288), (33, 1000, 4640), (64, 500, 8224)])
def test_every_form(m, n, k):
    """Sizes around the changes of the kernel: x whole in LDS or not, tiles of 16 to 256 rows, 16 to 64 tokens, several tiles per workgroup; both
    formats in one call."""
    rng = np.random.default_rng(m + n + k)
    x, xd = tokens(rng, m, k)
    ws = [weight(rng, n, k, snip.FP4), weight(rng, n // 3 + 1, k, snip.FP8)]
    for (q, w), y in zip(ws, snip.snip_gemv(x, [q for q, _ in ws], out_dtype=snip.OUT_FP32)):
        check(y, xd, w)


@pytest.mark.parametrize("fmt", [snip.FP4, snip.FP8])
@pytest.mark.parametrize("m,n,k", [(1, 4096, 4096), (5, 40, 96), (16, 1000, 1056), (40, 300, 512), (64, 80, 11008)])
def test_small_integers_are_exact(m, n, k, fmt):
    """x in -2 .. 2, weights 0, 1, 2, 4 (times a scale of 1 or 2) and their negatives: sums of at most 2^18 2^4 < 2^24."""
    rng = np.random.default_rng(k)
    xd = rng.integers(-2, 3, (m, k)).astype(np.float64)
    pick = rng.integers(0, 7, (n, k))
    v = np.array([0, 1, 2, 4, -1, -2, -4.])[pick]
    if fmt == snip.FP4:
        nib = np.array([0, 2, 4, 6, 10, 12, 14], np.uint8)[pick]
        codes = torch.from_numpy(nib[:, 0::2] | nib[:, 1::2] << 4)
    else:
        codes = torch.from_numpy(v).to(torch.float8_e4m3fn).view(torch.uint8)
    byte = rng.integers(127, 129, (n, k // 32)).astype(np.uint8)
    w = v * np.repeat(2.0 ** (byte - 127.0), 32, 1)
    q = snip.QTensor(codes.cuda(), torch.from_numpy(byte).cuda(), n, k, fmt)
    y = snip.snip_gemv(torch.from_numpy(xd).to(torch.bfloat16).cuda(), [q], out_dtype=snip.OUT_FP32)[0]
    assert np.array_equal(y.double().cpu().numpy(), xd @ w.T)


@pytest.mark.parametrize("m", [1, 20])
def test_weights_that_share_their_input(m):
    """19 weights of different widths and both formats, one of them empty: more than a launch takes; each as if alone."""
    rng = np.random.default_rng(m)
    x, xd = tokens(rng, m, 416)
    ws = [weight(rng, n, 416, f) for n, f in zip([16, 1, 33, 128, 250, 0, 64, 31, 5, 16, 48, 1000, 17, 2, 3, 129, 64, 8, 40], [0, 1] * 10)]
    ys = snip.snip_gemv(x, [q for q, _ in ws], out_dtype=snip.OUT_FP32)
    for y, (q, w) in zip(ys, ws):
        assert y.shape == (m, q.rows)
        if q.rows:
            check(y, xd, w)
            assert torch.equal(y, snip.snip_gemv(x, [q], out_dtype=snip.OUT_FP32)[0])
    assert snip.snip_gemv(x, []) == []
    assert snip.snip_gemv(x[:0], [ws[0][0]])[0].shape == (0, 16)


def test_what_quantize_makes():
    """The path of a program: bf16 weights quantized along their rows."""
    gen = torch.Generator(device="cuda").manual_seed(1)
    wt = (torch.randn(520, 1024, generator=gen, device="cuda") * 0.02).bfloat16()
    x = torch.randn(3, 1024, generator=gen, device="cuda").bfloat16()
    for fmt in (snip.FP4, snip.FP8):
        q = snip.snip_quantize(wt, fmt, snip.ROW)
        if fmt == snip.FP4:
            c = q.codes.cpu().numpy()
            nib = np.stack((c & 15, c >> 4), 2).reshape(520, 1024)
            v = np.where(nib & 8, -1, 1) * GRID4[nib & 7]
        else:
            v = q.codes.cpu().view(torch.float8_e4m3fn).double().numpy()
        check(snip.snip_gemv(x, [q])[0], x.double().cpu().numpy(), v * np.repeat(2.0 ** (q.scales.cpu().numpy() - 127.0), 32, 1))


@pytest.mark.parametrize("fmt", [snip.FP4, snip.FP8])
def test_scales_at_the_ends(fmt):
    """The lowest and highest scales, zeros under the lowest one, and the byte that is no number."""
    rng = np.random.default_rng(7)
    n, k = 40, 224
    x, xd = tokens(rng, 5, k)
    q, w = weight(rng, n, k, fmt)
    q.scales[1] = 2
    q.scales[2] = 0
    q.codes[2] = 0                                 # what quantize writes for a block of zeros
    q.scales[3] = 250 - (8 if fmt == snip.FP8 else 2)
    q.scales[4, 3] = 255
    per = 16 if fmt == snip.FP4 else 32
    q.codes[4, 3 * per:4 * per] = 0                # what quantize writes for a block with a NaN
    q.scales[5, 6] = 255
    y = snip.snip_gemv(x, [q], out_dtype=snip.OUT_FP32)[0].cpu().numpy()
    assert np.isnan(y[:, [4, 5]]).all()
    assert np.isfinite(np.delete(y, [4, 5], 1)).all() and (y[:, 2] == 0).all()


def test_scaled_rows():
    """A row's scale bytes raised or lowered by d multiply its outputs by 2^d exactly, down to the subnormal numbers and up to the largest."""
    rng = np.random.default_rng(8)
    x, xd = tokens(rng, 4, 256)
    for fmt in (snip.FP4, snip.FP8):
        q, w = weight(rng, 32, 256, fmt)
        y = snip.snip_gemv(x, [q], out_dtype=snip.OUT_FP32)[0].double()
        for d in (-100, 90):
            r = snip.QTensor(q.codes, (q.scales.int() + d).to(torch.uint8), 32, 256, fmt)
            assert torch.equal(snip.snip_gemv(x, [r], out_dtype=snip.OUT_FP32)[0].double(), y * 2.0 ** d)


def test_infinite_and_missing_numbers_stay_in_their_token():
    rng = np.random.default_rng(9)
    for k in (96, 4096):
        x, xd = tokens(rng, 20, k)
        q, w = weight(rng, 50, k, snip.FP4)
        x[3, k - 1] = float("inf")
        x[18, 0] = float("nan")
        y = snip.snip_gemv(x, [q], out_dtype=snip.OUT_FP32)[0]
        keep = [i for i in range(20) if i not in (3, 18)]
        check(y[keep], xd[keep], w)
        assert torch.isnan(y[18]).all() and not torch.isfinite(y[3]).any()


def test_codes_beyond_2_31_bytes():
    n, k = 66000, 65536
    q = snip.QTensor(torch.randint(0, 256, (n, k // 2), dtype=torch.uint8, device="cuda"), torch.full((n, k // 32), 127, dtype=torch.uint8, device="cuda"), n, k, snip.FP4)
    x = torch.randint(-2, 3, (2, k), device="cuda").bfloat16()
    y = snip.snip_gemv(x, [q], out_dtype=snip.OUT_FP32)[0]
    for rows in (slice(0, 4), slice(65534, 65540), slice(n - 4, n)):
        c = q.codes[rows].cpu().numpy()
        nib = np.stack((c & 15, c >> 4), 2).reshape(-1, k)
        assert np.array_equal(y[:, rows].double().cpu().numpy(), x.double().cpu().numpy() @ (np.where(nib & 8, -1, 1) * GRID4[nib & 7]).T)


def test_other_stream_and_graph():
    rng = np.random.default_rng(10)
    x, _ = tokens(rng, 3, 2048)
    ws = [weight(rng, n, 2048, f)[0] for n, f in ((2048, snip.FP4), (256, snip.FP8), (256, snip.FP4))]
    a = snip.snip_gemv(x, ws)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    b = snip.snip_gemv(x, ws, stream=side)
    side.synchronize()
    assert all(torch.equal(p, q) for p, q in zip(a, b))
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        snip.snip_gemv(x, ws, b)
    for _ in range(3):
        for t in b:
            t.zero_()
        g.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(p, q) for p, q in zip(a, b))


def test_refusals():
    x = torch.zeros((4, 64), dtype=torch.bfloat16, device="cuda")
    q = snip.alloc_qtensor(16, 64, snip.FP4)
    status = lambda *a, **k: pytest.raises(snip.SnipError, snip.snip_gemv, *a, **k).value.status  # noqa: E731
    assert status(x, [snip.alloc_qtensor(16, 96, snip.FP4)]) == 4                    # another contraction extent
    assert status(x[:, :40], [snip.alloc_qtensor(16, 64, snip.FP4)]) == 2
    assert status(torch.zeros((4, 68), dtype=torch.bfloat16, device="cuda")[:, :64], [q]) == 4
    assert status(x, [q], [torch.zeros((4, 17), dtype=torch.bfloat16, device="cuda")[:, :16]]) == 4
    bad = snip.QTensor(q.codes, q.scales, 16, 64, 3)
    assert status(x, [bad]) == 3
    for out in ([], [torch.zeros((3, 16), dtype=torch.bfloat16, device="cuda")], [torch.zeros((4, 16), dtype=torch.float16, device="cuda")], [torch.zeros((4, 16), dtype=torch.bfloat16)]):
        with pytest.raises(ValueError):
            snip.snip_gemv(x, [q], out)
    with pytest.raises(ValueError):
        snip.snip_gemv(x.float(), [q])
    with pytest.raises(TypeError):
        snip.snip_gemv(x, 3, [])
