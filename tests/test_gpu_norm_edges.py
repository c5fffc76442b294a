"""The norm where its sums are delicate: squares below the float range, and rows of millions of like values, whose
roundings do not cancel; and with so many rows that a block takes several, one after another.

Tolerances are those of test_gpu_norm, but for long rows: there a group of at most 8 elements is added in float and groups
in double, so that the roundings of a sum, LONG, do not grow with the row."""
import pytest
import test_gpu_norm as plain
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


# More rows than blocks (or waves with a row each) are launched, one to three and six groups a thread; six and eight groups of
# floats in a few rows.
MANY_ROWS = [(6500, 200), (6500, 1000), (4500, 1030), (2100, 2049), (1700, 5120), (1100, 9000), (1030, 12288)]


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [vcnn.F32, vcnn.BF16])
@pytest.mark.parametrize("rows,cols", MANY_ROWS + [(3, 9000), (3, 12288), (3, 16383)])
def test_many_rows_a_block(rows, cols, dtype):
    plain.test_forward(rows, cols, dtype, True, 0)
    plain.test_forward(rows, cols, dtype, False, 1)
    plain.test_eight_bits(rows, cols, dtype, 1)
    plain.test_backward(rows, cols, dtype, True)


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [vcnn.F32, vcnn.BF16])
@pytest.mark.parametrize("rows,cols", [(6500, 200), (2100, 2049), (1700, 5120)])
def test_many_rows_a_block_in_place(rows, cols, dtype):
    """The next row is on its way while a block's row is written: both in one tensor."""
    x, r, gain = tensor(91, rows, cols, dtype), tensor(92, rows, cols, dtype), dev(gain_of(93, cols))
    xd, rd = dev(x), dev(r)
    h, y, s = torch.empty_like(xd), torch.empty_like(xd), torch.empty(rows, device=DEV)
    vcnn.rmsnorm_fwd(dtype, rows, cols, plain.EPS, xd, rd, gain, h, y, s)
    assert torch.equal(h.cpu(), (x.float() + r.float()).to(x.dtype))
    q, q8 = (torch.empty(rows, cols, dtype=torch.int8, device=DEV) for _ in range(2))
    s8 = torch.empty(rows, device=DEV)
    vcnn.rmsnorm_fwd_i8(dtype, rows, cols, plain.EPS, xd, rd, gain, torch.empty_like(xd), q, s8)
    for which in ("h is x", "h is residual", "y is x"):
        a, b = xd.clone(), rd.clone()
        ho = {"h is x": a, "h is residual": b}.get(which, torch.empty_like(a))
        yo = a if which == "y is x" else torch.empty_like(a)
        vcnn.rmsnorm_fwd(dtype, rows, cols, plain.EPS, a, b, gain, ho, yo, None)
        assert torch.equal(ho, h) and torch.equal(yo, y), which
        if which != "y is x":
            a, b = xd.clone(), rd.clone()
            ho = a if which == "h is x" else b
            vcnn.rmsnorm_fwd_i8(dtype, rows, cols, plain.EPS, a, b, gain, ho, q8, s8)
            assert torch.equal(ho, h) and torch.equal(q8, q), which
    a = xd.clone()
    vcnn.rmsnorm_fwd(dtype, rows, cols, plain.EPS, a, None, gain, None, a, None)
    y0 = torch.empty_like(a)
    vcnn.rmsnorm_fwd(dtype, rows, cols, plain.EPS, xd, None, gain, None, y0, None)
    assert torch.equal(a, y0)
    dy, up = dev(tensor(94, rows, cols, dtype)), dev(tensor(95, rows, cols, dtype))
    dh = torch.empty_like(dy)
    vcnn.rmsnorm_bwd(dtype, rows, cols, h, gain, s, dy, up, dh, None)
    for which in ("dy", "above"):
        a, b = dy.clone(), up.clone()
        vcnn.rmsnorm_bwd(dtype, rows, cols, h, gain, s, a, b, a if which == "dy" else b, None)
        assert torch.equal(a if which == "dy" else b, dh), which
