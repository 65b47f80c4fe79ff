"""Corners of the norm, optimizer and few-token calls: rows that end inside a round of loads, scales at the ends of their range, dtypes,
what holds the tensors of a call, calls without the gains' gradient, large tensors' forms."""
import numpy as np
import pytest
import torch

from paper_2602_01410_amd import snip

pytestmark = pytest.mark.gpu

# tokens, rows, columns whose last spans lie behind the row's end, in each form of the few-token kernel; the last one in the small one
BEHIND = [(1, 40, 3328), (1, 9000, 3328), (3, 40, 5120), (16, 40, 11008), (16, 5000, 14336), (20, 300, 5120), (33, 1000, 4640), (48, 300, 11008), (64, 40, 3328),
          (64, 9000, 3328), (5, 40, 224)]


@pytest.mark.parametrize("fmt", [snip.FP4, snip.FP8])
@pytest.mark.parametrize("m,n,k", BEHIND)
def test_large_scales_beside_large_codes_in_the_last_block(m, n, k, fmt):
    """Small codes under scales close to the largest (2^125 and 2^120 each) and, in the last block, the largest code under a scale of 2^-7: all weights
    are finite, and so are the outputs; the last block is below a unit in the last place of them.  k equal positive products are within k 2^-24 of their sum.
    Row 1 has an infinite weight in its last block, row 2 a scale byte that is no number."""
    small, large, byte, per = (0x11, 0x77, 253, 16) if fmt == snip.FP4 else (0x38, 0x7E, 247, 32)
    codes = torch.full((n, k // 32 * per), small, dtype=torch.uint8, device="cuda")
    scales = torch.full((n, k // 32), byte, dtype=torch.uint8, device="cuda")
    codes[:, -per:] = large
    scales[:, -1] = 120
    scales[1, -1] = 254
    scales[2, 0] = 255
    x = (torch.arange(m, device="cuda").float() + 1).mul(2.0 ** -20)[:, None].expand(m, k).bfloat16().contiguous()
    y = snip.snip_gemv(x, [snip.QTensor(codes, scales, n, k, fmt)], out_dtype=snip.OUT_FP32)[0].double().cpu().numpy()
    want = x[:, 0].double().cpu().numpy() * (k - 32) * 2.0 ** (125 if fmt == snip.FP4 else 120)
    assert (y[:, 1] == np.inf).all() and np.isnan(y[:, 2]).all()
    rest = np.delete(y, (1, 2), 1)
    assert (np.abs(rest / want[:, None] - 1) <= k * 2.0 ** -24).all()


def test_longest_rows():
    """k = 2^31 - 32: x is 4 GB, its last chunk ends 32 elements before 2^31.  Few elements of x are not zero, so that the sums are exact."""
    n, k = 2, (1 << 31) - 32
    codes = torch.full((n, k // 2), 0x11, dtype=torch.uint8, device="cuda")              # 0.5
    codes[1] = 0xA2                                                                      # 1 and -1 in turn
    scales = torch.full((n, k // 32), 127, dtype=torch.uint8, device="cuda")
    x = torch.zeros((1, k), dtype=torch.bfloat16, device="cuda")
    at = [0, 5, 4097, k // 2, k - 32768, k - 33, k - 1]
    for i, c in enumerate(at):
        x[0, c] = 2.0 ** i
    y = snip.snip_gemv(x, [snip.QTensor(codes, scales, n, k, snip.FP4)], out_dtype=snip.OUT_FP32)[0].cpu().tolist()
    assert y == [[sum(2.0 ** i for i in range(len(at))) / 2, sum((-1.0) ** (c % 2) * 2.0 ** i for i, c in enumerate(at))]]


def test_more_rows_than_workgroups():
    """2^22 + 3 rows of 16 waves each (69 GB) are 2^32 threads and more; the rows of a second turn have their own norms."""
    rows, cols = (1 << 22) + 3, 8200
    x = torch.zeros((rows, cols), dtype=torch.bfloat16, device="cuda")
    at = torch.tensor([0, 1, (1 << 21) - 1, 1 << 21, (1 << 21) + 1, (1 << 22) - 1, 1 << 22, rows - 1], device="cuda")
    x[at] = (torch.arange(len(at), device="cuda") + 1).bfloat16()[:, None]
    rstd = torch.full((rows,), -1.0, device="cuda")
    w = torch.ones(cols, device="cuda")
    # no output but rstd: through the C call, since the binding's always delivers y or codes
    assert snip._lib().snip_rms_norm(x.data_ptr(), rows, cols, cols, None, 0, w.data_ptr(), 1, 1.0, 0, None, 0, rstd.data_ptr(), None, 0, None, None, None) == 0
    torch.cuda.synchronize()
    want = 1 / np.sqrt(1 + (np.arange(len(at)) + 1.0) ** 2)
    assert (np.abs(rstd[at].double().cpu().numpy() / want - 1) <= 3e-6).all()
    rstd[at] = 1.0
    assert bool((rstd == 1).all())
    del x
    torch.cuda.empty_cache()


def test_more_columns_than_a_launch_sums():
    """Gains' gradients of 2^27 + 8 columns, 32 a workgroup of 1024 threads: more than 2^32 threads."""
    cols = (1 << 27) + 8
    gen = torch.Generator(device="cuda").manual_seed(5)
    dy, h = (torch.randint(-8, 9, (2, cols), generator=gen, device="cuda").bfloat16() for _ in range(2))
    w = torch.ones(cols, dtype=torch.bfloat16, device="cuda")
    _, dw = snip.snip_rms_norm_backward(dy, h, w, torch.tensor([1.0, 0.5], device="cuda"))
    want = dy[0].float() * h[0].float() + dy[1].float() * h[1].float() * 0.5                    # (few bits: exact)
    assert torch.equal(dw, want)
    del dy, h, dw, want
    torch.cuda.empty_cache()


@pytest.mark.parametrize("rows,cols,smaller", [(512, 1024, [(256, 1024), (200, 1024), (257, 1017), (512, 520)]), (4096, 8192, [(4096, 8191), (1500, 4097), (700, 1001)]),
                                               (1100, 16384, [(1100, 8191), (1024, 4095), (513, 16377)])])
def test_workspace_of_the_largest_matrix_serves_the_others(rows, cols, smaller):
    workspace = torch.empty(snip.rms_norm_workspace_bytes(rows, cols), dtype=torch.uint8, device="cuda")
    for r, c in smaller:
        dy, h = (torch.ones((r, (c + 7) // 8 * 8), dtype=torch.bfloat16, device="cuda")[:, :c] for _ in range(2))
        _, dw = snip.snip_rms_norm_backward(dy, h, torch.ones(c, device="cuda"), torch.ones(r, device="cuda"), workspace=workspace)
        assert bool((dw == r).all())


def test_half_precision_is_not_bf16():
    """fp16 has bf16's size; its bits mean other numbers.  Bit patterns in 16-bit integers are taken as bf16's, as before."""
    x = torch.randn(32, 64, device="cuda")
    h, b, w, rstd = x.half(), x.bfloat16(), torch.ones(64, device="cuda"), torch.ones(32, device="cuda")
    q = snip.alloc_qtensor(32, 64, snip.FP8)
    weight = snip.snip_quantize(b, snip.FP8, snip.ROW)
    stats = torch.zeros(3, dtype=torch.float64, device="cuda")
    ws = snip.alloc_workspace(32, 64, x.device)
    for bad in (lambda: snip.snip_rms_norm(h, w, 1e-5), lambda: snip.snip_rms_norm(b, w, 1e-5, residual=h), lambda: snip.snip_rms_norm(b, w, 1e-5, residual=b, sum=h),
                lambda: snip.snip_rms_norm(b, w, 1e-5, y=h), lambda: snip.snip_rms_norm_backward(h, b, w, rstd), lambda: snip.snip_rms_norm_backward(b, h, w, rstd),
                lambda: snip.snip_rms_norm_backward(b, b, w, rstd, dsum=h), lambda: snip.snip_rms_norm_backward(b, b, w, rstd, dx=h), lambda: snip.snip_gemv(h, [weight]),
                lambda: snip.snip_quantize(h, snip.FP8), lambda: snip.snip_quantize(h, snip.FP8, out=q), lambda: snip.snip_quantize_both(h, snip.FP8, snip.FP4),
                lambda: snip.snip_quant_error_stats(h, snip.ROW, snip.NO_OVERFLOW, stats, workspace=ws)):
        with pytest.raises(ValueError):
            bad()
    for bits in (torch.int16, torch.uint16):
        assert torch.equal(snip.snip_rms_norm(b.view(bits), w, 1e-5).y, snip.snip_rms_norm(b, w, 1e-5).y)
        assert torch.equal(snip.snip_quantize(b.view(bits), snip.FP8).codes, snip.snip_quantize(b, snip.FP8).codes)


def test_tensors_of_an_iterable_are_held_until_the_call_is_launched():
    """Nobody but the iterable has them; what the end of the last reference does (here: it zeroes an input, on the same stream) comes after the
    launch."""
    class Param(snip.AdamwTensor):
        def __del__(self):
            self.grad.zero_()

    class Weight(snip.QTensor):
        def __del__(self):
            self.codes.zero_()

    n, params = 5000, []

    def tensors():
        for _ in range(3):
            t = Param(*(torch.full((n,), v, device="cuda") for v in (1.0, 1.0, 0.0, 0.0)))
            params.append((t.param, t.m, t.grad))
            yield t
            del t

    snip.snip_adamw_step(tensors(), 1e-2, 0.75, 0.75, 1e-8, 1)
    for p, m, g in params:
        assert bool((g == 0).all()) and bool((m == 0.25).all()) and bool(((p - 0.99).abs() < 1e-5).all())

    def weights(codes):
        for c in codes:
            yield Weight(c, torch.full((40, 2), 127, dtype=torch.uint8, device="cuda"), 40, 64, snip.FP4)

    codes = [torch.full((40, 32), 0x22, dtype=torch.uint8, device="cuda") for _ in range(2)]
    outs = [torch.zeros((4, 40), device="cuda") for _ in codes]
    x = torch.ones((4, 64), device="cuda").bfloat16()
    snip.snip_gemv(x, weights(codes), outs)
    assert all(bool((c == 0).all()) for c in codes) and all(bool((y == 64).all()) for y in outs)


@pytest.mark.parametrize("rows,cols", [(0, 64), (3, 13), (512, 512), (700, 1024), (96, 2048), (96, 4096), (40, 8192), (20, 16384), (7, 16391), (5, 32768)])
def test_gradient_without_that_of_the_gains(rows, cols):
    """In every form: dx has the bytes of the call that delivers both."""
    gen = torch.Generator(device="cuda").manual_seed(rows + cols)
    dy, h, ds = (torch.randn((rows, (cols + 7) // 8 * 8), generator=gen, device="cuda").bfloat16()[:, :cols] for _ in range(3))
    w, rstd = torch.randn(cols, generator=gen, device="cuda"), torch.rand(rows, generator=gen, device="cuda")
    both, dw = snip.snip_rms_norm_backward(dy, h, w, rstd, dsum=ds)
    dx, none = snip.snip_rms_norm_backward(dy, h, w, rstd, dsum=ds, gains=False)
    assert none is None and dw.shape == (cols,) and torch.equal(dx, both)
    with pytest.raises(ValueError):
        snip.snip_rms_norm_backward(dy, h, w, rstd, dweight=dw, gains=False)


@pytest.mark.parametrize("dsum", [False, True])
@pytest.mark.parametrize("cols", [504, 512, 1016, 1024, 2040, 2048, 4088, 4096, 8184, 8192, 16376, 16384])
def test_gradient_of_tensors_beyond_the_last_level_cache(cols, dsum):
    """The smallest calls whose tensors exceed 256 MB, which read past the caches, in every number of waves; all rows and all columns.  dx as in
    test_gpu_rms_norm.py: its parts are off by 2 DELTA at most before the rounding to bf16.  dweight: a term is added at most rows / 256 times in a lane, three times between
    waves and 16 between workgroups, a factor and a product are rounded before and the sum behind the doubles after that."""
    delta = 3e-6
    rows = (256 << 20) // (cols * (8 if dsum else 6)) + 1
    gen = torch.Generator(device="cuda").manual_seed(cols + dsum)
    dy, h, ds = (torch.randn((rows, cols), generator=gen, device="cuda").bfloat16() for _ in range(3))
    h[rows // 3] = 0
    w, rstd = 1 + 0.2 * torch.randn(cols, generator=gen, device="cuda"), 0.5 + torch.rand(rows, generator=gen, device="cuda")
    dx, dw = snip.snip_rms_norm_backward(dy, h, w, rstd, dsum=ds if dsum else None)
    total, magnitude = torch.zeros(cols, dtype=torch.float64, device="cuda"), torch.zeros(cols, dtype=torch.float64, device="cuda")
    step = (4 << 20) // cols
    for i in range(0, rows, step):
        d, x, r = dy[i:i + step].double(), h[i:i + step].double(), rstd[i:i + step].double()[:, None]
        g = d * w.double()
        ref = r * (g - x * r * r * (g * x).mean(1, keepdim=True))
        parts = r * (g.abs() + x.abs() * r * r * (g * x).abs().mean(1, keepdim=True))
        if dsum:
            ref, parts = ref + ds[i:i + step].double(), parts + ds[i:i + step].double().abs()
        got = dx[i:i + step].double()
        lo, hi = ((ref + e * parts).float().bfloat16().double() for e in (-2 * delta, 2 * delta))
        assert bool(((got >= lo) & (got <= hi)).all()), i
        t = d * x * r
        total += t.sum(0)
        magnitude += t.abs().sum(0)
    assert bool(((dw.double() - total).abs() <= (rows / 256 + 24) * 2.0 ** -24 * magnitude).all())


@pytest.mark.parametrize("fmt", [snip.FP4, snip.FP8])
@pytest.mark.parametrize("end", ["lowest", "highest"])
@pytest.mark.parametrize("m,n,k", [(5, 40, 224), (1, 50, 3328), (16, 9000, 3328), (16, 40, 11008), (40, 300, 4640), (64, 500, 4128)])
def test_values_at_the_ends_of_the_scales(m, n, k, end, fmt):
    """Weights below bf16's normal numbers (scale bytes 0 to 3: code 2^-127 ...) are rounded to its nearest subnormal one, 2^-134 off at most (FP4's, and
    FP8's from byte 3 on, are exact); those under the highest scales that keep all codes finite are exact.  x is scaled so that products and sums are normal."""
    from test_gpu_gemv import weight
    rng = np.random.default_rng(m * n + k)
    top = 253 if fmt == snip.FP4 else 247                        # from here on the largest code is infinite
    q, w = weight(rng, n, k, fmt, *((0, 4) if end == "lowest" else (top - 4, top)))
    x = torch.from_numpy(rng.standard_normal((m, k)).astype(np.float32) * np.float32(2.0 ** (60 if end == "lowest" else -60))).bfloat16()
    y = snip.snip_gemv(x.cuda(), [q], out_dtype=snip.OUT_FP32)[0].double().cpu().numpy()
    xd = x.double().numpy()
    room = k * 2.0 ** -24 * (np.abs(xd) @ np.abs(w.T)) + (np.abs(xd).sum(1)[:, None] * 2.0 ** -134 if end == "lowest" else 0)
    assert (np.abs(y - xd @ w.T) <= room).all()


@pytest.mark.parametrize("beta1", [0.5, 0.9, 0.99])
def test_8_bit_moments_stop_where_the_header_says(beta1):
    """Moments of 1, gradients from then on between -1 and 1 that do not change, one of 1 in each group, which keeps the scale: m comes as close as half
    the distance of its numbers, |m| / 16 or 2^-10 of the scale, over 1 - beta1.  Moments of 32 bits get there."""
    n = 128 * 64
    g = torch.linspace(-1, 1, n, device="cuda")
    g[::128] = 1.0
    small, exact = (snip.alloc_adamw_state(torch.zeros(n, device="cuda"), g, bits) for bits in (8, 32))
    small.m.fill_(0x7E)
    small.m_scale.fill_(1 / 448)
    exact.m.fill_(1.0)
    for step in range(1, 2001):
        snip.snip_adamw_step([small, exact], 0.0, beta1, 0.95, 1e-8, step, seed=step)
    scale = small.m_scale.repeat_interleave(128)
    m = small.m.view(torch.float8_e4m3fn).float() * scale
    assert bool((scale * 448 - 1 < 1e-5).all())
    assert bool(((g - m).abs() <= torch.maximum(m.abs() / 16, scale * 2.0 ** -10) / (1 - beta1) * 1.001).all())
    assert bool(((g - exact.m).abs() < 1e-5).all())
