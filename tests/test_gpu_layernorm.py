"""Layer norm (forward with dropout and the residual, backward) against plain forms in 64 bits.

Tolerances.  A sum of a row is a tree: at most 32 elements a thread kept in registers (rows of more than 16384 elements: in double),
six exchanges in a wave, at most 16 waves, and a few roundings more of what is done with it: depth() roundings of 2^-24 of the sum
of magnitudes.  The mean is taken twice, the second time about the first, so its error is that of the deviations' sum.  A result is
then rounded once to its type.  A column's sum goes over a block's rows, 64 parts and six pairs."""
import pytest
import torch

from paper_1501_07338_amd import vcnn
from test_gpu_dropout import factors, generator
from test_gpu_norm import DEV, EPS, SHAPES, TYPES, U, Guarded, depth, dev, gain_of, half_step, tensor

SEED, STEP, SITE = 0x123456789abcdef, 7, 4


def column_depth(rows):
    return rows / 128 + 64 + 16


def reference(h, gain, bias, eps=EPS):
    hd = h.double()
    mean = hd.mean(1)
    d = hd - mean[:, None]
    rstd = (d.square().mean(1) + eps).rsqrt()
    y = d * rstd[:, None] * gain.double() + (0 if bias is None else bias.double())
    return mean, rstd, y


def check_forward(h, gain, bias, got_y, got_mean, got_rstd, dtype, eps=EPS):
    rows, cols = h.shape
    mean, rstd, y = reference(h, gain, bias, eps)
    hd, n = h.double(), depth(cols)
    off = (hd - mean[:, None]).abs().mean(1) + n * U * hd.abs().mean(1)  # what the second sum adds up
    assert bool(((got_mean.double() - mean).abs() <= 2 * U * mean.abs() + n * U * off + 1e-40).all())
    assert float(((got_rstd.double() - rstd) / rstd).abs().max()) <= n * U
    zg = ((hd - mean[:, None]) * rstd[:, None] * gain.double()).abs()
    slack = n * U * (zg + gain.double().abs() * (off * rstd)[:, None]) + 2 * U * y.abs()
    assert bool(((got_y.double() - y).abs() <= 1.01 * (half_step(dtype) * y.abs() + slack) + 1e-40).all())


@pytest.mark.gpu
@pytest.mark.parametrize("offset", [0, 1])
@pytest.mark.parametrize("residual,p", [(False, 0.0), (True, 0.0), (False, 0.25), (True, 0.25)])
@pytest.mark.parametrize("dtype", [vcnn.F32, vcnn.BF16])
@pytest.mark.parametrize("rows,cols", SHAPES)
def test_forward(rows, cols, dtype, residual, p, offset):
    x, gain = tensor(1, rows, cols, dtype), gain_of(3, cols)
    r = tensor(2, rows, cols, dtype) if residual else None
    bias = gain_of(4, cols) - 1.0 if offset else None
    rng = generator(SEED, STEP)
    h, y = Guarded((rows, cols), x.dtype, offset), Guarded((rows, cols), x.dtype, offset)
    mean, rstd = Guarded((rows,), torch.float32), Guarded((rows,), torch.float32)
    stored = residual or p > 0
    vcnn.layernorm_fwd(dtype, rows, cols, EPS, p, rng if p else None, SITE, dev(x, offset), dev(r, offset), dev(gain, offset),
                       dev(bias, offset), h.t if stored else None, y.t, mean.t, rstd.t)
    read = x
    if p > 0:  # the same elements as the call of its own, and the same sums
        want = torch.empty(rows, cols, dtype=x.dtype, device=DEV)
        vcnn.dropout_fwd(dtype, rows, cols, p, rng, SITE, dev(x), dev(r), want)
        read = want.cpu()
        assert torch.equal(h.cpu(), read)
    elif residual:
        read = (x.float() + r.float()).to(x.dtype)
        assert torch.equal(h.cpu(), read)
    check_forward(read, gain, bias, y.cpu(), mean.cpu(), rstd.cpu(), dtype)


def gradients(h, gain, mean, rstd, dy, above, f):
    """In 64 bits from the mean and rstd that the call is given."""
    hd, d, g = h.double(), dy.double(), gain.double()
    z, t = (hd - mean.double()[:, None]) * rstd.double()[:, None], d * g
    dh = rstd.double()[:, None] * (t - t.mean(1, keepdim=True) - z * (t * z).mean(1, keepdim=True))
    size = rstd.double()[:, None] * (t.abs() + t.abs().mean(1, keepdim=True) + z.abs() * (t * z).abs().mean(1, keepdim=True))
    if above is not None:
        dh, size = dh + above.double(), size + above.double().abs()
    return dh, (dh if f is None else dh * f), (d * z).sum(0), d.sum(0), size, (d * z).abs().sum(0), d.abs().sum(0)


@pytest.mark.gpu
@pytest.mark.parametrize("offset", [0, 1])
@pytest.mark.parametrize("p", [0.0, 0.25])
@pytest.mark.parametrize("dtype", [vcnn.F32, vcnn.BF16])
@pytest.mark.parametrize("rows,cols", SHAPES)
def test_backward(rows, cols, dtype, p, offset):
    h, dy, gain = tensor(21, rows, cols, dtype), tensor(22, rows, cols, dtype, loud=False), gain_of(23, cols)
    above = tensor(24, rows, cols, dtype, loud=False) if offset else None
    mean, rstd, _ = reference(h, gain, None)
    mean, rstd = mean.float(), rstd.float()
    f = factors(rows, cols, p, SEED, STEP, SITE) if p else None
    wdh, wdx, wdg, wdb, size, sg, sb = gradients(h, gain, mean, rstd, dy, above, f)
    dh, dx = Guarded((rows, cols), h.dtype, offset), Guarded((rows, cols), h.dtype, offset)
    dg, db = Guarded((cols,), torch.float32, offset), Guarded((cols,), torch.float32, offset)
    ws = torch.full((vcnn.layernorm_workspace_bytes(rows, cols),), 0x5a, dtype=torch.uint8, device=DEV)
    args = (dtype, rows, cols, p, generator(SEED, STEP) if p else None, SITE, dev(h, offset), dev(gain, offset), dev(mean),
            dev(rstd), dev(dy, offset), dev(above, offset))
    vcnn.layernorm_bwd(*args, dh.t, dx.t if p else None, dg.t, db.t, ws)
    n = depth(cols)
    assert bool(((dh.cpu().double() - wdh).abs() <= 1.01 * half_step(dtype) * wdh.abs() + n * U * size + 1e-40).all())
    if p:
        assert bool(((dx.cpu().double() - wdx).abs() <= 1.01 * half_step(dtype) * wdx.abs() + 2 * n * U * size + 1e-40).all())
        assert bool((dx.cpu()[f == 0] == 0).all())
    assert bool(((dg.cpu().double() - wdg).abs() <= column_depth(rows) * U * sg + 1e-40).all())
    assert bool(((db.cpu().double() - wdb).abs() <= column_depth(rows) * U * sb + 1e-40).all())
    # the same bits again, each output alone too
    for k in range(4):
        if k == 1 and not p:
            continue
        alone = [None] * 4
        alone[k] = torch.full_like((dh, dx, dg, db)[k].t, 3.0)
        vcnn.layernorm_bwd(*args, *alone, ws if k > 1 else None)
        assert torch.equal(alone[k].cpu(), (dh, dx, dg, db)[k].cpu())


@pytest.mark.gpu
@pytest.mark.parametrize("cols", [5, 96, 1000, 17000])
def test_gradient_against_differences(cols):
    """sum(y dy) along a direction of h: the formula's values in 64 bits on both sides, and the kernel's gradient."""
    rows, e = 3, 1e-4
    h, dy, gain = tensor(31, rows, cols, vcnn.F32, loud=False), tensor(32, rows, cols, vcnn.F32, loud=False), gain_of(33, cols)
    way = torch.randn(rows, cols, generator=torch.Generator().manual_seed(34), dtype=torch.float64)
    mean, rstd, _ = reference(h, gain, None)
    dh = torch.empty(rows, cols, device=DEV)
    vcnn.layernorm_bwd(vcnn.F32, rows, cols, 0.0, None, 0, dev(h), dev(gain), dev(mean.float()), dev(rstd.float()), dev(dy), None,
                       dh, None, None, None)

    def cost(at):
        return float((reference(at, gain, None)[2] * dy.double()).sum())

    slope = (cost(h.double() + e * way) - cost(h.double() - e * way)) / (2 * e)
    *_, size, _, _ = gradients(h, gain, mean, rstd, dy, None, None)
    # the difference's own error: e^2 times a third derivative, of the order of the terms' sizes times rstd^2 |way|^2 ...
    own = 10 * e * e * float((size * way.abs()).sum()) * float((rstd ** 2).max()) * float(way.abs().max()) ** 2
    assert abs(float((dh.cpu().double() * way).sum()) - slope) <= depth(cols) * U * float((size * way.abs()).sum()) + own + 1e-8


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [vcnn.F32, vcnn.BF16])
@pytest.mark.parametrize("cols", [64, 1500, 5000, 20000])
def test_rows_of_all_kinds(cols, dtype):
    """Like values, means that dwarf the spread, values whose squares leave the float range at either end, infinities, NaN."""
    g = torch.Generator().manual_seed(41)
    base = torch.randn(cols, generator=g)
    kinds = [torch.full((cols,), 3.25), 1e4 + base, 1e-30 * base, 1e30 * base, -1e38 + 1e38 * base.clamp(-2, 2), torch.zeros(cols),
             base.clone(), base.clone(), base]
    x = torch.stack(kinds).to(TYPES[dtype])
    x[6, cols // 2], x[7, cols - 1] = float("inf"), float("nan")
    rows = x.shape[0]
    gain, bias = gain_of(42, cols), gain_of(43, cols)
    for eps in (1e-5, 1e-38):
        y, mean, rstd = Guarded((rows, cols), x.dtype), Guarded((rows,), torch.float32), Guarded((rows,), torch.float32)
        vcnn.layernorm_fwd(dtype, rows, cols, eps, 0.0, None, 0, dev(x), None, dev(gain), dev(bias), None, y.t, mean.t, rstd.t)
        got = y.cpu()
        assert bool(torch.isnan(got[6:8]).all())
        fine = [0, 1, 2, 3, 4, 5, 8]
        if eps == 1e-38:
            fine = [1, 2, 3, 4, 8]  # (at 1e19 a standard deviation the others' own roundings are all there is)
        assert bool(torch.isfinite(got[fine]).all())
        m, s, _ = reference(x[fine], gain, bias, float(torch.tensor(eps, dtype=torch.float32)))
        # rstd of a row of 1e38 is a float below the normal range: steps of 2^-149
        assert bool(((rstd.cpu()[fine].double() - s).abs() <= depth(cols) * U * s + 2.0 ** -149).all())
        wide = [i for i, k in enumerate(fine) if k != 4]
        at = [fine[i] for i in wide]
        check_forward(x[at], gain, bias, got[at], mean.cpu()[at], rstd.cpu()[at], dtype, float(torch.tensor(eps, dtype=torch.float32)))
    one = torch.empty(3, 1, device=DEV)
    vcnn.layernorm_fwd(vcnn.F32, 3, 1, EPS, 0.0, None, 0, dev(torch.tensor([[5.0], [-1e30], [0.0]])), None, dev(gain[:1]),
                       dev(bias[:1]), None, one, None, None)
    assert torch.equal(one.cpu(), bias[:1].expand(3, 1))


@pytest.mark.gpu
@pytest.mark.parametrize("rows,cols", [(5, 500), (700, 2049), (3, 20001)])
@pytest.mark.parametrize("dtype", [vcnn.F32, vcnn.BF16])
def test_in_place(rows, cols, dtype):
    x, r, gain, bias = tensor(51, rows, cols, dtype), tensor(52, rows, cols, dtype), gain_of(53, cols), gain_of(54, cols)
    rng, dg, db = generator(SEED, STEP), dev(gain), dev(bias)
    h, y = torch.empty_like(dev(x)), torch.empty_like(dev(x))
    mean, rstd = torch.empty(rows, device=DEV), torch.empty(rows, device=DEV)
    vcnn.layernorm_fwd(dtype, rows, cols, EPS, 0.2, rng, SITE, dev(x), dev(r), dg, db, h, y, mean, rstd)
    for inside in ("x", "residual"):
        px, pr, py = dev(x), dev(r), torch.empty_like(y)
        into = px if inside == "x" else pr
        if inside == "residual":
            py = px
        vcnn.layernorm_fwd(dtype, rows, cols, EPS, 0.2, rng, SITE, px, pr, dg, db, into, py, mean, rstd)
        assert torch.equal(into, h) and torch.equal(py, y)
    dy, above = dev(tensor(55, rows, cols, dtype)), dev(tensor(56, rows, cols, dtype))
    dh, dx = torch.empty_like(h), torch.empty_like(h)
    args = (dtype, rows, cols, 0.2, rng, SITE, h, dg, mean, rstd)
    vcnn.layernorm_bwd(*args, dy, above, dh, dx, None, None)
    for swap in (False, True):
        a, b = dy.clone(), above.clone()
        vcnn.layernorm_bwd(*args, a, b, b if swap else a, a if swap else b, None, None)
        assert torch.equal(b if swap else a, dh) and torch.equal(a if swap else b, dx)


@pytest.mark.gpu
def test_captured_forward_and_backward():
    """Replays under new inputs and steps, with eager calls on the same tensors between them."""
    rows, cols, dtype = 300, 1000, vcnn.BF16
    x, r, dy = (dev(tensor(s, rows, cols, dtype)) for s in (61, 62, 63))
    gain, bias, rng = dev(gain_of(64, cols)), dev(gain_of(65, cols)), generator(SEED, 0)
    ws = torch.empty(vcnn.layernorm_workspace_bytes(rows, cols), dtype=torch.uint8, device=DEV)

    def outputs():
        return [torch.empty_like(x) for _ in range(4)] + [torch.empty(n, device=DEV) for n in (rows, rows, cols, cols)]

    def step(o, advance):
        h, y, dh, dx, mean, rstd, dg, db = o
        vcnn.layernorm_fwd(dtype, rows, cols, EPS, 0.1, rng, SITE, x, r, gain, bias, h, y, mean, rstd)
        vcnn.layernorm_bwd(dtype, rows, cols, 0.1, rng, SITE, h, gain, mean, rstd, dy, None, dh, dx, dg, db, ws)
        if advance:
            vcnn.rng_advance(rng)

    o, want = outputs(), outputs()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step(o, True)
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step(o, True)
    for n in range(4):
        x.copy_(dev(tensor(70 + n, rows, cols, dtype)))
        step(want, False)
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(o, want))
        assert int(rng[1]) == n + 2


def test_refusals_need_no_gpu():
    lib, f = vcnn.lib(), 0x1000  # never dereferenced: validation fails first

    def fwd(dtype=vcnn.F32, rows=2, cols=8, eps=1e-5, p=0.0, rng=None, x=f, r=None, gain=f, h=None, y=f):
        return lib.vcnn_layernorm_fwd(dtype, rows, cols, eps, p, rng, 0, x, r, gain, None, h, y, None, None, None)

    assert fwd(rows=0) == vcnn.ERR_SHAPE and fwd(cols=0) == vcnn.ERR_SHAPE and fwd(dtype=9) == vcnn.ERR_UNSUPPORTED
    assert fwd(cols=(1 << 30) + 1) == vcnn.ERR_UNSUPPORTED
    for eps in (0.0, -1.0, float("nan"), float("inf")):
        assert fwd(eps=eps) == vcnn.ERR_UNSUPPORTED
    assert fwd(x=None) == vcnn.ERR_NULL and fwd(gain=None) == vcnn.ERR_NULL and fwd(y=None) == vcnn.ERR_NULL
    assert fwd(r=f) == vcnn.ERR_NULL  # h is written with a residual
    assert fwd(p=0.5, h=f) == vcnn.ERR_NULL and fwd(p=0.5, rng=f) == vcnn.ERR_NULL  # no generator; no h
    assert fwd(p=1.0, rng=f, h=f) == vcnn.ERR_UNSUPPORTED and fwd(p=0.5, rng=0x1001, h=f) == vcnn.ERR_UNSUPPORTED

    def bwd(rows=2, p=0.0, rng=None, h=f, mean=f, rstd=f, dy=f, dh=f, dx=None, dg=None, db=None, ws=None, nbytes=0):
        return lib.vcnn_layernorm_bwd(vcnn.F32, rows, 8, p, rng, 0, h, f, mean, rstd, dy, None, dh, dx, dg, db, ws, nbytes, None)

    need = vcnn.layernorm_workspace_bytes(2, 8)
    assert need >= 2 * 2 * 8 * 4
    assert bwd(rows=0) == vcnn.ERR_SHAPE and bwd(h=None) == vcnn.ERR_NULL and bwd(mean=None) == vcnn.ERR_NULL
    assert bwd(rstd=None) == vcnn.ERR_NULL and bwd(dy=None) == vcnn.ERR_NULL
    assert bwd(dx=0x2000) == vcnn.ERR_UNSUPPORTED  # no dropout
    assert bwd(p=0.5, rng=f, dx=f) == vcnn.ERR_UNSUPPORTED  # dh itself
    assert bwd(dg=f) == vcnn.ERR_WORKSPACE and bwd(db=f, ws=0x1100, nbytes=need - 1) == vcnn.ERR_WORKSPACE
    assert bwd(db=f, ws=0x1110, nbytes=need) == vcnn.ERR_WORKSPACE
    assert bwd(dh=None) == vcnn.OK  # nothing is wanted
    assert lib.vcnn_layernorm_workspace_bytes(2, 8, None) == vcnn.ERR_NULL
    assert lib.vcnn_layernorm_workspace_bytes(0, 8, None) != vcnn.OK
