"""The fully connected layer in 8-bit integers against whole-number sums.

Tolerance: the sum is exact; then it is rounded to float, so is the product of the scales, and so is the fused
multiplication and addition of the bias: three roundings of 2^-24 of |sum scale| + |bias|, an activation good to a few more
(tanh, the logistic function: 2^-21 of their result or of 1), and the rounding to y's type."""
import ctypes

import pytest
import torch

from paper_1501_07338_amd import vcnn
from test_gpu_norm import DEV, TYPES, Guarded, dev, half_step

U = 2.0 ** -24
# batch, in_f, out_f: one sample to many, one input to many, odd rows and rows of whole words, tiles that end inside, the
# kernel for few samples with one to four tiles of them, divided sums
SHAPES = [(1, 1, 1), (1, 16, 3), (1, 4096, 513), (2, 127, 18), (16, 128, 16), (17, 129, 33), (33, 1000, 100), (47, 515, 64),
          (64, 4097, 40), (65, 15, 7), (65, 17, 130), (65, 128, 128), (100, 1024, 257), (129, 2064, 130), (200, 4100, 300),
          (257, 272, 255), (128, 8192, 128), (300, 640, 9001)]


def make(seed, batch, k, out, full=False):
    g = torch.Generator().manual_seed(seed)
    low = -128 if full else -127
    x = torch.randint(low, 128, (batch, k), generator=g, dtype=torch.int8)
    w = torch.randint(low, 128, (out, k), generator=g, dtype=torch.int8)
    xs = (0.5 + torch.rand(batch, generator=g)) / 4000
    ws = (0.5 + torch.rand(out, generator=g)) / (4000 * k ** 0.5)
    return x, w, xs, ws, 0.3 * torch.randn(out, generator=g)


def reference(x, w, xs, ws, bias, act):
    s = (x.double() @ w.double().t()) * xs.double()[:, None] * ws.double()[None, :]  # (sums below 2^31: exact)
    size = s.abs()
    if bias is not None:
        s, size = s + bias.double(), size + bias.double().abs()
    y = {vcnn.ACT_NONE: lambda v: v, vcnn.ACT_RELU: lambda v: v.clamp(min=0), vcnn.ACT_TANH: torch.tanh,
         vcnn.ACT_SIGMOID: torch.sigmoid}[act](s)
    return y, size


def call(dtype, act, x, w, xs, ws, bias, workspace, offset=0):
    (batch, k), out = x.shape, w.shape[0]
    y = Guarded((batch, out), TYPES[dtype], offset)
    vcnn.fc_fwd_i8(dtype, batch, k, out, act, dev(x, offset), dev(xs), dev(w, offset), dev(ws), dev(bias), y.t, workspace)
    return y.cpu()


@pytest.mark.gpu
@pytest.mark.parametrize("offset", [0, 1])
@pytest.mark.parametrize("dtype", [vcnn.F32, vcnn.BF16])
@pytest.mark.parametrize("batch,k,out", SHAPES)
def test_against_exact_sums(batch, k, out, dtype, offset):
    need = vcnn.fc_i8_workspace_bytes(batch, k, out)
    for act, with_bias in ((vcnn.ACT_NONE, False), (vcnn.ACT_RELU, True), (vcnn.ACT_TANH, True), (vcnn.ACT_SIGMOID, False)):
        x, w, xs, ws, bias = make(batch + k + out, batch, k, out, full=act == vcnn.ACT_RELU)
        bias = bias if with_bias else None
        want, size = reference(x, w, xs, ws, bias, act)
        smooth = 0.0 if act in (vcnn.ACT_NONE, vcnn.ACT_RELU) else 8 * U
        got = call(dtype, act, x, w, xs, ws, bias, torch.empty(max(need, 256), dtype=torch.uint8, device=DEV), offset)
        off = (got.double() - want).abs()
        assert bool((off <= want.abs() * half_step(dtype) * 1.01 + size * 4 * U + smooth).all())
        # the same bits with no workspace, and with part of it
        for more in ([None, 256] if need else [None]):
            ws_t = None if more is None else torch.empty(more, dtype=torch.uint8, device=DEV)
            assert torch.equal(call(dtype, act, x, w, xs, ws, bias, ws_t, offset), got)


@pytest.mark.gpu
@pytest.mark.parametrize("offset", [0, 1])
@pytest.mark.parametrize("batch,k,out", [(1000, 112, 12300), (1000, 100, 12300), (770, 200, 16390)])
def test_large_tiles(batch, k, out, offset):
    """Enough tiles of 256 x 256, the last of them ragged on both sides."""
    x, w, xs, ws, bias = make(batch + k, batch, k, out)
    want, size = reference(x, w, xs, ws, bias, vcnn.ACT_RELU)
    for dtype in (vcnn.F32, vcnn.BF16):
        off = (call(dtype, vcnn.ACT_RELU, x, w, xs, ws, bias, None, offset).double() - want).abs()
        assert bool((off <= want.abs() * half_step(dtype) * 1.01 + size * 4 * U).all())


@pytest.mark.gpu
@pytest.mark.parametrize("batch", [1, 20, 64, 70, 260])
def test_every_sum_is_whole(batch):
    """Scales of one: floats of the sums themselves, below 2^24 with every bit; large ones at the longest rows."""
    k, out = 1000, 300
    x, w, _, _, _ = make(7, batch, k, out, full=True)
    one = torch.ones(max(batch, out))
    got = call(vcnn.F32, vcnn.ACT_NONE, x, w, one[:batch], one[:out], None, None)
    assert torch.equal(got.double(), x.double() @ w.double().t())
    k = 131071
    x, w = torch.full((batch, k), -128, dtype=torch.int8), torch.full((3, k), -128, dtype=torch.int8)
    w[1] = 127
    w[2, ::2] = 127
    got = call(vcnn.F32, vcnn.ACT_NONE, x, w, one[:batch], one[:3], None, None)
    want = (x[:1].double() @ w.double().t()).float().expand(batch, 3)
    assert torch.equal(got, want)


@pytest.mark.gpu
@pytest.mark.parametrize("batch", [3, 90])
def test_scales_that_are_not_numbers_stay_in_their_rows(batch):
    x, w, xs, ws, bias = make(9, batch, 200, 70)
    xs[1], ws[5], xs[2] = float("nan"), float("nan"), 0.0
    for act in (vcnn.ACT_NONE, vcnn.ACT_RELU):
        got = call(vcnn.F32, act, x, w, xs, ws, bias, None)
        nan = torch.zeros(batch, 70, dtype=torch.bool)
        nan[1], nan[:, 5] = True, True
        assert torch.equal(torch.isnan(got), nan)
        keep = torch.ones(70, dtype=torch.bool)
        keep[5] = False
        assert torch.equal(got[2][keep], (bias.clamp(min=0) if act else bias)[keep])


@pytest.mark.gpu
def test_normalised_and_answered():
    """The norm's 8-bit output through an 8-bit layer against the same layer in floats: a hidden layer, its norm, the residual."""
    batch, k, out = 96, 800, 500
    g = torch.Generator().manual_seed(3)
    x, r, gain = torch.randn(batch, k, generator=g), torch.randn(batch, k, generator=g), 1 + 0.2 * torch.randn(k, generator=g)
    w, bias = torch.randn(out, k, generator=g) * (2.0 / k) ** 0.5, 0.1 * torch.randn(out, generator=g)
    h, q, s = torch.empty(batch, k, device=DEV), torch.empty(batch, k, dtype=torch.int8, device=DEV), torch.empty(batch, device=DEV)
    wq, ws = torch.empty(out, k, dtype=torch.int8, device=DEV), torch.empty(out, device=DEV)
    y, rstd, z, yf = (torch.empty(n, device=DEV) for n in ((batch, out), (batch,), (batch, k), (batch, out)))
    xd, rd, gd, wd, bd = (dev(t) for t in (x, r, gain, w, bias))
    vcnn.quant_rows_i8(vcnn.F32, out, k, wd, wq, ws)
    vcnn.rmsnorm_fwd_i8(vcnn.F32, batch, k, 1e-6, xd, rd, gd, h, q, s)
    vcnn.fc_fwd_i8(vcnn.F32, batch, k, out, vcnn.ACT_RELU, q, s, wq, ws, bd, y)
    vcnn.rmsnorm_fwd(vcnn.F32, batch, k, 1e-6, xd, rd, gd, h, z, rstd)
    vcnn.fc_fwd(vcnn.F32, batch, k, out, vcnn.ACT_RELU, z, wd, bd, yf)
    torch.cuda.synchronize()
    # an operand is off by at most half a step a / 127 an element: of a sum, |z| dw + |w| dz + dz dw over the row
    dz, dw = s[:, None] / 2, ws[None, :] / 2
    bound = z.abs().sum(1, keepdim=True) * dw + wd.abs().sum(1)[None, :] * dz + k * dz * dw
    assert bool(((y - yf).abs() <= bound * 1.001).all())
    # and what the integers say is what the layer gave
    want, size = reference(q.cpu(), wq.cpu(), s.cpu(), ws.cpu(), bias, vcnn.ACT_RELU)
    assert bool(((y.cpu().double() - want).abs() <= size * 4 * U + want.abs() * U).all())


@pytest.mark.gpu
@pytest.mark.parametrize("batch,k,out", [(5, 700, 90), (128, 8192, 128)])
def test_on_a_stream_of_its_own_and_in_a_graph(batch, k, out):
    x, w, xs, ws, bias = (dev(t) for t in make(5, batch, k, out))
    work = torch.empty(max(256, vcnn.fc_i8_workspace_bytes(batch, k, out)), dtype=torch.uint8, device=DEV)
    y = torch.empty(batch, out, dtype=torch.bfloat16, device=DEV)

    def go():
        vcnn.fc_fwd_i8(vcnn.BF16, batch, k, out, vcnn.ACT_NONE, x, xs, w, ws, bias, y, work)

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        go()
    torch.cuda.synchronize()
    want = y.clone()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        go()
    for _ in range(3):
        y.zero_()
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(y, want)


def test_refusals_need_no_gpu():
    lib = vcnn.lib()
    f = 0x1000  # never dereferenced: validation fails first

    def go(dtype=vcnn.F32, batch=4, k=8, out=4, act=0, p=(f,) * 5, ws=None, n=0):
        return lib.vcnn_fc_fwd_i8(dtype, batch, k, out, act, p[0], p[1], p[2], p[3], None, p[4], ws, n, None)

    for name in ("batch", "k", "out"):
        for v in (0, -3):
            assert go(**{name: v}) == vcnn.ERR_SHAPE
    assert go(k=131072) == vcnn.ERR_UNSUPPORTED and "32 bits" in vcnn.last_error()
    assert go(batch=2 ** 31 - 1, out=2 ** 31 - 1) == vcnn.ERR_UNSUPPORTED
    assert go(dtype=9) == vcnn.ERR_UNSUPPORTED and go(act=4) == vcnn.ERR_UNSUPPORTED and go(act=-1) == vcnn.ERR_UNSUPPORTED
    for i in range(5):
        assert go(p=tuple(None if j == i else f for j in range(5))) == vcnn.ERR_NULL
    assert go(ws=0x1010, n=256) == vcnn.ERR_WORKSPACE
    assert go(ws=0x1010, n=0, act=9) == vcnn.ERR_UNSUPPORTED
    assert lib.vcnn_fc_i8_workspace_bytes(4, 8, 4, None) == vcnn.ERR_NULL
    assert lib.vcnn_fc_i8_workspace_bytes(4, 0, 4, ctypes.byref(ctypes.c_size_t())) == vcnn.ERR_SHAPE
    assert vcnn.fc_i8_workspace_bytes(1, 4096, 4096) == 0
