"""The root-mean-square norm (forward, backward, 8-bit output) and the quantisation of rows against plain forms in 64 bits.

Tolerances.  A sum of a row is a tree: at most 32 elements a thread kept in registers (rows of more than 16384 elements:
one in 4096 of them or 8192), six exchanges in a wave, at most 16 waves - DEPTH roundings of 2^-24 of the sum of
magnitudes, and a few more of what is done with it (EXTRA).  A result is then rounded once to its type."""
import ctypes

import numpy as np
import pytest
import torch

from paper_1501_07338_amd import vcnn

DEV = "cuda:0"
EPS = 1e-6
U = 2.0 ** -24
EXTRA = 12
SHAPES = [(1, 1), (1, 2), (3, 7), (5, 64), (2, 500), (128, 500), (4, 513), (7, 1024), (3, 1025), (2, 4097), (5, 5120),
          (3, 8191), (2, 16384), (2, 16391), (3, 40001), (1300, 33), (4100, 200), (700, 2049)]
TYPES = {vcnn.F32: torch.float32, vcnn.BF16: torch.bfloat16}


def depth(cols):
    return (32 if cols <= 16384 else cols // 4096 + 8) + 6 + 16 + EXTRA


def half_step(dtype):
    return torch.finfo(TYPES[dtype]).eps / 2


def tensor(seed, rows, cols, dtype, loud=True):
    g = torch.Generator().manual_seed(seed)
    x = torch.randn(rows, cols, generator=g) * torch.exp(0.5 * torch.randn(rows, 1, generator=g))
    if loud:
        x[:, torch.randint(0, cols, (max(1, cols // 64),), generator=g)] *= 12.0
    return x.to(TYPES[dtype])


def gain_of(seed, cols):
    return 1.0 + 0.3 * torch.randn(cols, generator=torch.Generator().manual_seed(seed))


def dev(t, offset=0):
    """On the GPU, `offset` elements behind the start of an allocation."""
    if t is None:
        return None
    b = torch.zeros(t.numel() + offset, dtype=t.dtype, device=DEV)
    b[offset:].copy_(t.reshape(-1))
    return b[offset:].view(t.shape)


class Guarded:
    """An output with a band of known bytes around it."""

    def __init__(self, shape, dtype, offset=0):
        self.n = int(np.prod(shape))
        self.pad = 64 + offset
        self.all = torch.zeros(self.n + 2 * 64 + offset, dtype=dtype, device=DEV)
        self.all.view(torch.uint8).fill_(0x5a)
        self.t = self.all[self.pad:self.pad + self.n].view(shape)

    def cpu(self):
        torch.cuda.synchronize()
        edge = torch.cat([self.all[:self.pad], self.all[self.pad + self.n:]]).view(torch.uint8)
        assert bool((edge == 0x5a).all()), "bytes around the output were written"
        return self.t.cpu()


def reference(x, r, gain):
    h = x if r is None else (x.float() + r.float()).to(x.dtype)
    hd = h.double()
    rstd = (hd.square().mean(1) + EPS).rsqrt()
    return h, rstd, hd * rstd[:, None] * gain.double()


def integers(u):
    """127 u / a of 32-bit values, in 64 bits: the products are exact and the quotient is rounded once."""
    a = u.abs().amax(1, keepdim=True)
    q = torch.where(a > 0, torch.round(u.double() * 127 / a.double()), 0.0)
    return q, a[:, 0].double()


@pytest.mark.gpu
@pytest.mark.parametrize("offset", [0, 1])
@pytest.mark.parametrize("residual", [False, True])
@pytest.mark.parametrize("dtype", [vcnn.F32, vcnn.BF16])
@pytest.mark.parametrize("rows,cols", SHAPES)
def test_forward(rows, cols, dtype, residual, offset):
    x, gain = tensor(1, rows, cols, dtype), gain_of(3, cols)
    r = tensor(2, rows, cols, dtype) if residual else None
    h, rstd, y = reference(x, r, gain)
    ho, yo, so = Guarded((rows, cols), x.dtype, offset), Guarded((rows, cols), x.dtype, offset), Guarded((rows,), torch.float32)
    vcnn.rmsnorm_fwd(dtype, rows, cols, EPS, dev(x, offset), dev(r, offset), dev(gain, offset), ho.t if residual else None,
                     yo.t, so.t)
    if residual:
        assert torch.equal(ho.cpu(), h)  # one addition, rounded once
    assert float(((so.cpu().double() - rstd) / rstd).abs().max()) <= depth(cols) * U
    off = (yo.cpu().double() - y).abs()
    assert bool((off <= y.abs() * (half_step(dtype) + depth(cols) * U) * 1.01 + 1e-40).all())


@pytest.mark.gpu
@pytest.mark.parametrize("offset", [0, 1])
@pytest.mark.parametrize("dtype", [vcnn.F32, vcnn.BF16])
@pytest.mark.parametrize("rows,cols", SHAPES)
def test_eight_bits(rows, cols, dtype, offset):
    x, r, gain = tensor(11, rows, cols, dtype), tensor(12, rows, cols, dtype), gain_of(13, cols)
    x[rows // 2] = 0.0
    for res in (None, r):
        h, rstd, _ = reference(x, res, gain)
        want, a = integers(h.float() * gain)
        q, s = Guarded((rows, cols), torch.int8, offset), Guarded((rows,), torch.float32)
        ho = Guarded((rows, cols), x.dtype, offset)
        vcnn.rmsnorm_fwd_i8(dtype, rows, cols, EPS, dev(x, offset), dev(res, offset), dev(gain), ho.t, q.t, s.t)
        assert torch.equal(q.cpu().double(), want)
        scale = a * rstd / 127
        assert bool(((s.cpu().double() - scale).abs() <= scale * depth(cols) * U).all())
        if res is not None:
            assert torch.equal(ho.cpu(), h)
    want, a = integers(x.float())
    q, s = Guarded((rows, cols), torch.int8, offset), Guarded((rows,), torch.float32)
    vcnn.quant_rows_i8(dtype, rows, cols, dev(x, offset), q.t, s.t)
    assert torch.equal(q.cpu().double(), want)
    assert bool(((s.cpu().double() - a / 127).abs() <= a / 127 * 2 * U).all())


@pytest.mark.gpu
def test_ties_go_to_even_and_the_border_is_exact():
    x = torch.arange(-127, 128, dtype=torch.float32)[None, :] / 2.0
    x = torch.cat([x, torch.tensor([[127.0]])], 1)  # a = 127: the quotients are the elements, half of them ties
    near = torch.cat([torch.nextafter(x, torch.full_like(x, 1e9)), torch.nextafter(x, torch.full_like(x, -1e9))])
    near[:, -1] = 127.0
    rng = torch.randn(64, 8192, generator=torch.Generator().manual_seed(5))
    small = rng[:4] * 1e-37  # 127 / a leaves the float range
    for u in (x, near, rng, small, rng[:4] * 1e-42, rng[:4] * 1e37):
        rows, cols = u.shape
        q, s = Guarded((rows, cols), torch.int8), Guarded((rows,), torch.float32)
        vcnn.quant_rows_i8(vcnn.F32, rows, cols, dev(u), q.t, s.t)
        want, a = integers(u)
        assert torch.equal(q.cpu().double(), want)
        # (a scale below the smallest normal float is a multiple of 2^-149)
        assert bool(((s.cpu().double() - a / 127).abs() <= a / 127 * 2 * U + 2.0 ** -149).all())


def reference_bwd(h, gain, dy, above):
    hd, t, d = h.double(), dy.double() * gain.double(), dy.double()
    rstd = (hd.square().mean(1) + EPS).rsqrt()[:, None]
    z = hd * rstd
    dh = rstd * (t - z * (t * z).mean(1, keepdim=True))
    size = rstd * (t.abs() + z.abs() * (t * z).abs().mean(1, keepdim=True))
    if above is not None:
        dh, size = dh + above.double(), size + above.double().abs()
    return dh, size, (d * z).sum(0), (d * z).abs().sum(0)


@pytest.mark.gpu
@pytest.mark.parametrize("above", [False, True])
@pytest.mark.parametrize("dtype", [vcnn.F32, vcnn.BF16])
@pytest.mark.parametrize("rows,cols", SHAPES)
def test_backward(rows, cols, dtype, above):
    offset = 1 if above else 0
    h, dy, gain = tensor(21, rows, cols, dtype), tensor(22, rows, cols, dtype, loud=False), gain_of(23, cols)
    up = tensor(24, rows, cols, dtype) if above else None
    dh, size, dg, dg_size = reference_bwd(h, gain, dy, up)
    rstd = (h.double().square().mean(1) + EPS).rsqrt().float().to(DEV)
    dho, dgo = Guarded((rows, cols), h.dtype, offset), Guarded((cols,), torch.float32)
    ws = torch.empty(vcnn.rmsnorm_workspace_bytes(rows, cols), dtype=torch.uint8, device=DEV)
    args = [dev(h, offset), dev(gain), rstd, dev(dy, offset), dev(up, offset)]
    vcnn.rmsnorm_bwd(dtype, rows, cols, *args, dho.t, dgo.t, ws)
    got = dho.cpu()
    off = (got.double() - dh).abs()
    assert bool((off <= dh.abs() * half_step(dtype) * 1.01 + size * depth(cols) * U + 1e-40).all())
    # a block's rows in turn, four waves, at most 512 blocks sixteen at a time, sixteen sums; two roundings an element
    terms = -(-rows // 512) + 4 + 32 + 16 + EXTRA
    first = dgo.cpu()
    assert bool(((first.double() - dg).abs() <= dg_size * terms * U + 1e-40).all())
    # either alone gives the same bits, and so does every run
    alone, galone = Guarded((rows, cols), h.dtype, offset), Guarded((cols,), torch.float32)
    vcnn.rmsnorm_bwd(dtype, rows, cols, *args, alone.t, None)
    vcnn.rmsnorm_bwd(dtype, rows, cols, *args, None, galone.t, ws)
    assert torch.equal(alone.cpu(), got) and torch.equal(galone.cpu(), first)


@pytest.mark.gpu
def test_gradients_against_differences():
    rows, cols = 3, 37
    h, gain, dy = tensor(31, rows, cols, vcnn.F32), gain_of(32, cols), tensor(33, rows, cols, vcnn.F32)

    def loss(hd, gd):
        return float((dy.double() * hd * (hd.square().mean(1, keepdim=True) + EPS).rsqrt() * gd).sum())

    hd, gd, step = h.double(), gain.double(), 1e-6
    dh, dg = torch.zeros(rows, cols, dtype=torch.float64), torch.zeros(cols, dtype=torch.float64)
    for i in range(rows * cols):
        e = torch.zeros(rows * cols, dtype=torch.float64)
        e[i] = step
        dh.view(-1)[i] = (loss(hd + e.view(rows, cols), gd) - loss(hd - e.view(rows, cols), gd)) / (2 * step)
    for i in range(cols):
        e = torch.zeros(cols, dtype=torch.float64)
        e[i] = step
        dg[i] = (loss(hd, gd + e) - loss(hd, gd - e)) / (2 * step)
    y, rstd = torch.empty(rows, cols, device=DEV), torch.empty(rows, device=DEV)
    vcnn.rmsnorm_fwd(vcnn.F32, rows, cols, EPS, dev(h), None, dev(gain), None, y, rstd)
    dho, dgo = torch.empty(rows, cols, device=DEV), torch.empty(cols, device=DEV)
    ws = torch.empty(vcnn.rmsnorm_workspace_bytes(rows, cols), dtype=torch.uint8, device=DEV)
    vcnn.rmsnorm_bwd(vcnn.F32, rows, cols, dev(h), dev(gain), rstd, dev(dy), None, dho, dgo, ws)
    # the differences are good to step^2 and to 2^-52 |loss| / step: some 1e-8; the kernel to 70 roundings of a float
    assert float((dho.cpu().double() - dh).abs().max()) <= 1e-5 * float(dh.abs().max())
    assert float((dgo.cpu().double() - dg).abs().max()) <= 1e-5 * float(dg.abs().max())


@pytest.mark.gpu
@pytest.mark.parametrize("cols", [40, 2900, 20000])
def test_rows_that_leave_the_range(cols):
    """Magnitudes whose squares are no floats, infinities, NaN and zeros stay in their own rows."""
    rows = 9
    x, gain = tensor(41, rows, cols, vcnn.F32), gain_of(42, cols)
    x[1] *= 1e30
    x[2] *= 1e-30
    x[3] = 0.0
    x[4, cols // 2] = float("inf")
    x[5, cols - 1] = float("nan")
    x[6] = 3.0e38
    y, s = Guarded((rows, cols), torch.float32), Guarded((rows,), torch.float32)
    vcnn.rmsnorm_fwd(vcnn.F32, rows, cols, EPS, dev(x), None, dev(gain), None, y.t, s.t)
    _, rstd, want = reference(x, None, gain)
    y, s = y.cpu().double(), s.cpu().double()
    for i in (0, 1, 2, 3, 6, 7, 8):
        assert bool(((y[i] - want[i]).abs() <= want[i].abs() * 2 * depth(cols) * U + 1e-40).all()), i
    assert bool(torch.isnan(y[5]).all()) and bool(torch.isnan(s[5]))
    assert float(s[4]) == 0.0 and bool(torch.isnan(y[4, cols // 2])) and float(y[4].nan_to_num(0.0).abs().max()) == 0.0
    q, sc = Guarded((rows, cols), torch.int8), Guarded((rows,), torch.float32)
    x[6] = 1.5e38  # (h * gain stays finite)
    vcnn.rmsnorm_fwd_i8(vcnn.F32, rows, cols, EPS, dev(x), None, dev(gain), None, q.t, sc.t)
    want, a = integers(torch.nan_to_num(x * gain, 0.0, 0.0, 0.0))
    q, sc = q.cpu().double(), sc.cpu().double()
    for i in (0, 1, 2, 3, 6, 7, 8):
        assert torch.equal(q[i], want[i]), i
        full = float(a[i]) * float((x[i].double().square().mean() + EPS).rsqrt()) / 127
        assert abs(float(sc[i]) - full) <= full * depth(cols) * U + 2.0 ** -149
    for i in (4, 5):
        assert bool(torch.isnan(sc[i])) and float(q[i].abs().max()) == 0.0
    q, sc = Guarded((rows, cols), torch.int8), Guarded((rows,), torch.float32)
    vcnn.quant_rows_i8(vcnn.F32, rows, cols, dev(x), q.t, sc.t)
    q, sc = q.cpu(), sc.cpu()
    assert bool(torch.isnan(sc[4])) and bool(torch.isnan(sc[5])) and int(q[4:6].abs().max()) == 0
    assert float(sc[3]) == 0.0 and int(q[3].abs().max()) == 0 and bool(torch.isfinite(sc[[0, 1, 2, 6, 7, 8]]).all())


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [vcnn.F32, vcnn.BF16])
@pytest.mark.parametrize("cols", [96, 2500, 16500])
def test_in_place(cols, dtype):
    rows = 6
    x, r, gain = tensor(51, rows, cols, dtype), tensor(52, rows, cols, dtype), dev(gain_of(53, cols))
    xd, rd = dev(x), dev(r)
    h, y, s = torch.empty_like(xd), torch.empty_like(xd), torch.empty(rows, device=DEV)
    vcnn.rmsnorm_fwd(dtype, rows, cols, EPS, xd, rd, gain, h, y, s)
    for which in ("h is x", "h is residual", "y is x"):
        a, b = xd.clone(), rd.clone()
        ho = {"h is x": a, "h is residual": b}.get(which, torch.empty_like(a))
        yo = a if which == "y is x" else torch.empty_like(a)
        vcnn.rmsnorm_fwd(dtype, rows, cols, EPS, a, b, gain, ho, yo, None)
        assert torch.equal(ho, h) and torch.equal(yo, y), which
    dy, up = dev(tensor(54, rows, cols, dtype)), dev(tensor(55, rows, cols, dtype))
    dh = torch.empty_like(dy)
    vcnn.rmsnorm_bwd(dtype, rows, cols, h, gain, s, dy, up, dh, None)
    for which in ("dy", "above"):
        a, b = dy.clone(), up.clone()
        vcnn.rmsnorm_bwd(dtype, rows, cols, h, gain, s, a, b, a if which == "dy" else b, None)
        assert torch.equal(a if which == "dy" else b, dh), which


@pytest.mark.gpu
def test_on_a_stream_of_its_own_and_in_a_graph():
    rows, cols, dtype = 37, 1800, vcnn.BF16
    x, r, gain, dy = (dev(t) for t in (tensor(61, rows, cols, dtype), tensor(62, rows, cols, dtype), gain_of(63, cols),
                                       tensor(64, rows, cols, dtype)))
    h, y, dh = (torch.empty_like(x) for _ in range(3))
    q, qs = torch.empty(rows, cols, dtype=torch.int8, device=DEV), torch.empty(rows, device=DEV)
    s, dg = torch.empty(rows, device=DEV), torch.empty(cols, device=DEV)
    ws = torch.empty(vcnn.rmsnorm_workspace_bytes(rows, cols), dtype=torch.uint8, device=DEV)

    def chain():
        vcnn.rmsnorm_fwd(dtype, rows, cols, EPS, x, r, gain, h, y, s)
        vcnn.rmsnorm_fwd_i8(dtype, rows, cols, EPS, x, r, gain, h, q, qs)
        vcnn.rmsnorm_bwd(dtype, rows, cols, h, gain, s, dy, None, dh, dg, ws)

    outs = (h, y, s, q, qs, dh, dg)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        chain()
    torch.cuda.synchronize()
    want = [t.clone() for t in outs]
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        chain()
    for _ in range(3):
        for t in outs:
            t.zero_()
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(outs, want))


def test_refusals_need_no_gpu():
    lib = vcnn.lib()
    f = 0x1000  # never dereferenced: validation fails first
    e = ctypes.c_float(EPS)
    bad = [((0, 4), vcnn.ERR_SHAPE), ((4, 0), vcnn.ERR_SHAPE), ((-1, 4), vcnn.ERR_SHAPE), ((1, (1 << 30) + 1), vcnn.ERR_UNSUPPORTED)]
    for (rows, cols), status in bad:
        assert lib.vcnn_rmsnorm_fwd(vcnn.F32, rows, cols, e, f, None, f, None, f, f, None) == status
        assert lib.vcnn_rmsnorm_fwd_i8(vcnn.F32, rows, cols, e, f, None, f, None, f, f, None) == status
        assert lib.vcnn_rmsnorm_bwd(vcnn.F32, rows, cols, f, f, f, f, None, f, None, None, 0, None) == status
        assert lib.vcnn_quant_rows_i8(vcnn.F32, rows, cols, f, f, f, None) == status
        assert lib.vcnn_rmsnorm_workspace_bytes(rows, cols, ctypes.byref(ctypes.c_size_t())) == status
    for value in (0.0, -1e-6, float("inf"), float("nan")):
        assert lib.vcnn_rmsnorm_fwd(vcnn.F32, 2, 4, ctypes.c_float(value), f, None, f, None, f, f, None) == vcnn.ERR_UNSUPPORTED
    assert lib.vcnn_rmsnorm_fwd(7, 2, 4, e, f, None, f, None, f, f, None) == vcnn.ERR_UNSUPPORTED
    for missing in range(3):
        p = [f, f, f]
        p[missing] = None
        assert lib.vcnn_rmsnorm_fwd(vcnn.F32, 2, 4, e, p[0], None, p[1], None, p[2], None, None) == vcnn.ERR_NULL
        assert lib.vcnn_rmsnorm_fwd_i8(vcnn.F32, 2, 4, e, p[0], None, p[1], None, p[2], f, None) == vcnn.ERR_NULL
        assert lib.vcnn_quant_rows_i8(vcnn.F32, 2, 4, *p, None) == vcnn.ERR_NULL
    assert lib.vcnn_rmsnorm_fwd(vcnn.F32, 2, 4, e, f, f, f, None, f, f, None) == vcnn.ERR_NULL  # a residual needs h
    assert lib.vcnn_rmsnorm_fwd_i8(vcnn.F32, 2, 4, e, f, None, f, None, f, None, None) == vcnn.ERR_NULL
    for missing in range(4):
        p = [f] * 4
        p[missing] = None
        assert lib.vcnn_rmsnorm_bwd(vcnn.F32, 2, 4, *p, None, f, None, None, 0, None) == vcnn.ERR_NULL
    need = vcnn.rmsnorm_workspace_bytes(2, 4)
    assert need == 32
    for ws, n in ((None, 0), (0x1010, need), (0x1100, need - 1)):
        assert lib.vcnn_rmsnorm_bwd(vcnn.F32, 2, 4, f, f, f, f, None, f, f, ws, n, None) == vcnn.ERR_WORKSPACE
    assert lib.vcnn_rmsnorm_bwd(vcnn.F32, 2, 4, f, f, f, f, None, None, None, None, 0, None) == vcnn.OK  # nothing asked for
    assert lib.vcnn_rmsnorm_workspace_bytes(2, 4, None) == vcnn.ERR_NULL
