"""The norm where its sums are delicate: squares below the float range, and rows of millions of like values, whose
roundings do not cancel.

Tolerances are those of test_gpu_norm, but for long rows: there a group of at most 8 elements is added in float and groups
in double, so that the roundings of a sum, LONG, do not grow with the row."""
import pytest
import torch

from paper_1501_07338_amd import vcnn
from test_gpu_norm import DEV, EXTRA, TYPES, U, Guarded, depth, dev, gain_of, half_step, tensor

LONG = 8 + EXTRA


@pytest.mark.gpu
@pytest.mark.parametrize("eps", [1e-40, 2.0 ** -149, 1e-36])
@pytest.mark.parametrize("cols", [40, 2900, 20000])
def test_squares_below_the_float_range(cols, eps):
    """eps may be any positive float: beside one this small, the squares of small rows count."""
    eps = float(torch.tensor(eps, dtype=torch.float32))
    size = torch.tensor([1.0, 1e-17, 1e-19, 1e-20, 3e-22, 1e-23, 1e-30, 0.0])
    rows = len(size)
    x, gain = tensor(71, rows, cols, vcnn.F32) * size[:, None], gain_of(72, cols)
    rstd = (x.double().square().mean(1) + eps).rsqrt()
    y, s = Guarded((rows, cols), torch.float32), Guarded((rows,), torch.float32)
    vcnn.rmsnorm_fwd(vcnn.F32, rows, cols, eps, dev(x), None, dev(gain), None, y.t, s.t)
    assert bool(((s.cpu().double() - rstd).abs() <= rstd * depth(cols) * U).all())
    want = x.double() * rstd[:, None] * gain.double()
    assert bool(((y.cpu().double() - want).abs() <= want.abs() * (depth(cols) + 2) * U + 1e-40).all())
    q, s = Guarded((rows, cols), torch.int8), Guarded((rows,), torch.float32)
    vcnn.rmsnorm_fwd_i8(vcnn.F32, rows, cols, eps, dev(x), None, dev(gain), None, q.t, s.t)
    scale = (x * gain).abs().amax(1).double() * rstd / 127
    assert bool(((s.cpu().double() - scale).abs() <= scale * depth(cols) * U + 2.0 ** -149).all())


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [vcnn.F32, vcnn.BF16])
@pytest.mark.parametrize("cols", [64 * 224 * 224, 16 * 131 * 131 + 5])
def test_long_rows_of_like_values(cols, dtype):
    """The activations of a convolution as one row: all of them 1.1 (and one row with a few negative ones)."""
    rows, eps = 2, 1e-6
    h = torch.full((rows, cols), 1.1).to(TYPES[dtype])
    h[1, ::7] = -0.7
    dy, gain = torch.full_like(h, 0.3), torch.full((cols,), 0.9)
    dy[1, ::5] = 0.8
    hd, t = h.double(), dy.double() * gain.double()
    rstd = (hd.square().mean(1) + eps).rsqrt()
    s, y = Guarded((rows,), torch.float32), Guarded((rows, cols), h.dtype)
    vcnn.rmsnorm_fwd(dtype, rows, cols, eps, dev(h), None, dev(gain), None, y.t, s.t)
    assert bool(((s.cpu().double() - rstd).abs() <= rstd * LONG * U).all())
    want = hd * rstd[:, None] * gain.double()
    assert bool(((y.cpu().double() - want).abs() <= want.abs() * (half_step(dtype) * 1.01 + LONG * U)).all())
    q, s8 = Guarded((rows, cols), torch.int8), Guarded((rows,), torch.float32)
    vcnn.rmsnorm_fwd_i8(dtype, rows, cols, eps, dev(h), None, dev(gain), None, q.t, s8.t)
    scale = (h.float() * gain).abs().amax(1).double() * rstd / 127
    assert bool(((s8.cpu().double() - scale).abs() <= scale * LONG * U).all())
    z = hd * rstd[:, None]
    want = rstd[:, None] * (t - z * (t * z).mean(1, keepdim=True))  # (like values cancel: the error is that of the terms)
    size = rstd[:, None] * (t.abs() + z.abs() * (t * z).abs().mean(1, keepdim=True))
    dh, dg = Guarded((rows, cols), h.dtype), Guarded((cols,), torch.float32)
    ws = torch.empty(vcnn.rmsnorm_workspace_bytes(rows, cols), dtype=torch.uint8, device=DEV)
    vcnn.rmsnorm_bwd(dtype, rows, cols, dev(h), dev(gain), rstd.float().to(DEV), dev(dy), None, dh.t, dg.t, ws)
    off = (dh.cpu().double() - want).abs()
    assert bool((off <= want.abs() * half_step(dtype) * 1.01 + size * LONG * U + 1e-40).all())
    want = (dy.double() * z).sum(0)
    assert bool(((dg.cpu().double() - want).abs() <= (dy.double() * z).abs().sum(0) * LONG * U).all())


@pytest.mark.gpu
def test_gain_gradient_of_more_columns_than_a_grid_is_wide():
    """2^26 columns and a few: sixteen a block of 1024 threads would be 2^32 threads and more in one dimension."""
    rows, cols = 2, (1 << 26) + 37
    g = torch.Generator(device=DEV).manual_seed(81)
    h = torch.randn(rows, cols, device=DEV, generator=g).to(torch.bfloat16)
    dy = torch.randn(rows, cols, device=DEV, generator=g).to(torch.bfloat16)
    gain, rstd = torch.ones(cols, device=DEV), torch.tensor([0.7, 1.9], device=DEV)
    dg = Guarded((cols,), torch.float32)
    ws = torch.empty(vcnn.rmsnorm_workspace_bytes(rows, cols), dtype=torch.uint8, device=DEV)
    vcnn.rmsnorm_bwd(vcnn.BF16, rows, cols, h, gain, rstd, dy, None, None, dg.t, ws)
    dg.cpu()
    for a in range(0, cols, 1 << 24):
        part = slice(a, a + (1 << 24))
        terms = dy[:, part].double() * h[:, part].double() * rstd.double()[:, None]
        assert bool(((dg.t[part].double() - terms.sum(0)).abs() <= terms.abs().sum(0) * 4 * U).all())
