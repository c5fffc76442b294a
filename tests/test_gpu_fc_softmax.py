"""The softmax cost of a fully connected layer with many classes, and its gradients, against plain forms in 64 bits.

Tolerances, from the number of roundings.  U = 2^-24.  A sum of n products in float takes at most n roundings of the sum of
magnitudes; the matrix cores add 16 or 32 products a step and may cut instead of rounding, which counts twice.  An error e of a logit
is an error e of a probability's logarithm, and so is one of the logarithm of the sum.  In bfloat16 dx is made from one term of the
difference, dw from three, or two from 4096 samples on.  A bfloat16 has 8 significant bits: its steps between 1 and 2 are 2^-7, a rounding is off by at most half of
one, 2^-8 of the value, that of what a first term leaves by 2^-8 of 2^-8, 2^-16, and a third one by 2^-24."""
import pytest
import torch

from paper_1501_07338_amd import vcnn
from test_gpu_norm import DEV, TYPES, U, Guarded, dev, half_step

IGNORE = -100
SHAPES = [(1, 1, 1), (1, 8, 10), (3, 7, 5), (5, 64, 10), (128, 500, 10), (64, 100, 1000), (130, 129, 257), (257, 64, 300),
          (300, 1032, 520), (70, 33, 4099), (513, 256, 2049), (17, 96, 20000), (700, 200, 16400), (16, 300, 5000), (9, 1030, 777),
          (2, 5, 70000), (40, 72, 17000), (64, 260, 130), (2500, 40, 300), (2100, 100, 90), (33, 2000, 65), (600, 500, 5000), (100, 3, 70)]
LARGE = [(2048, 6144, 300), (200, 2050, 6200), (1025, 40, 33000), (5000, 3, 9000), (200000, 5, 9), (70000, 130, 12),
         (5, 1000, 14000), (16, 703, 6100), (9, 1024, 7500)]


def inputs(batch, in_f, classes, dtype, ignored=0.2, seed=1):
    g = torch.Generator().manual_seed(seed)
    w = (torch.randn(classes, in_f, generator=g) * 1.5 / in_f ** 0.5).to(TYPES[dtype])
    labels = torch.randint(0, classes, (batch,), generator=g, dtype=torch.int32)
    x = torch.randn(batch, in_f, generator=g) + 8 * torch.rand(batch, 1, generator=g) * w.float()[labels.long()] / 1.5
    if ignored and batch > 1:
        labels[torch.rand(batch, generator=g) < ignored] = IGNORE
        labels[0] = int(torch.randint(0, classes, (), generator=g))
    return x.to(TYPES[dtype]), w, 0.5 * torch.randn(classes, generator=g), labels


def plain(x, w, bias, labels):
    """(loss, each, dx, dw, dbias, d) and bounds on what the float sums may leave in them, in 64 bits on the GPU."""
    x, w, labels = x.to(DEV).double(), w.to(DEV).double(), labels.to(DEV).long()
    bias = torch.zeros(w.shape[0], dtype=torch.float64, device=DEV) if bias is None else bias.to(DEV).double()
    counted = labels != IGNORE
    x = torch.where(counted[:, None], x, 0.0)
    wt = w.t().contiguous()
    z = x @ wt + bias
    lse = torch.logsumexp(z, 1)
    at = torch.where(counted, labels, 0)
    zl = z.gather(1, at[:, None])[:, 0]
    count = max(1, int(counted.sum()))
    each = torch.where(counted, lse - zl, 0.0)
    p = torch.exp(z - lse[:, None])
    d = p.clone()
    d.scatter_add_(1, at[:, None], torch.full_like(d[:, :1], -1.0))
    d *= counted[:, None]
    p = p * counted[:, None]
    out = dict(loss=each.sum() / count, each=each, dx=d @ w / count, dw=d.t().contiguous() @ x / count, db=d.sum(0) / count)
    # errors
    batch, in_f, classes = x.shape[0], x.shape[1], w.shape[0]
    steps = lambda n: 2 * (n + 16)  # noqa: E731  roundings of a sum of n products
    ez = steps(in_f) * U * (x.abs() @ wt.abs() + bias.abs()) + 2 * U * z.abs()
    es = (classes / 128 + 100) * U  # a tile's sums, the tiles' one after another, the exponentials' own errors
    worst = ez.amax(1)
    le = worst + es + 2 * U * lse.abs()
    eeach = counted * (le + ez.gather(1, at[:, None])[:, 0] + 2 * U * (lse.abs() + zl.abs()))
    ep = p * (ez + le[:, None] + 4 * U * (z.abs() + lse.abs()[:, None]) + 4 * U) + U * d.abs()
    bounds = dict(each=eeach, loss=eeach.sum() / count + (batch / 512 + 30) * U * out["loss"])
    aw, ax, ad = w.abs(), x.abs(), d.abs()

    def gradients(terms_dx, terms_dw):
        bounds["dx"] = (ep + (terms_dx + steps(classes) * U) * ad) @ aw / count + 4 * U * out["dx"].abs()
        bounds["dw"] = (ep + (terms_dw + steps(batch) * U) * ad).t().contiguous() @ ax / count + 4 * U * out["dw"].abs()
        bounds["db"] = (ep + steps(batch) * U * ad).sum(0) / count + 4 * U * out["db"].abs()
    return out, bounds, gradients


def run(dtype, x, w, bias, labels, want="dx dw db each", workspace=None, offset=0, part=None):
    batch, in_f, classes = x.shape[0], x.shape[1], w.shape[0]
    wants = want.split()
    t = TYPES[dtype]
    outs = {"loss": Guarded((1,), torch.float32)}
    for name, shape, kind in (("dx", (batch, in_f), t), ("dw", (classes, in_f), torch.float32), ("db", (classes,), torch.float32),
                              ("each", (batch,), torch.float32)):
        if name in wants:
            outs[name] = Guarded(shape, kind, offset)
    grads = any(n in wants for n in ("dx", "dw", "db"))
    if part is None:
        nbytes = vcnn.fc_softmax_loss_workspace_bytes(dtype, batch, in_f, classes, grads)
    else:
        nbytes = vcnn.fc_softmax_loss_workspace_bytes(dtype, part, in_f, classes, grads) + 4 * batch + 256
    ws = torch.full((nbytes + 1024,), 0xff, dtype=torch.uint8, device=DEV)  # floats of it are NaN
    to = lambda n: outs[n].t if n in outs else None  # noqa: E731
    vcnn.fc_softmax_loss(dtype, batch, in_f, classes, dev(x, offset), dev(w), dev(bias, offset), dev(labels), IGNORE, outs["loss"].t,
                         to("each"), to("dx"), to("dw"), to("db"), ws[:nbytes])
    got = {n: o.cpu() for n, o in outs.items()}
    assert bool((ws[nbytes:] == 0xff).all()), "bytes behind the workspace were written"
    return got


def check(dtype, got, out, bounds, gradients):
    bf = dtype == vcnn.BF16
    gradients(2.0 ** -8 if bf else 0.0, 0.0 if not bf else 2.0 ** -24 if out["each"].numel() < 4096 else 2.0 ** -16)
    for name, v in got.items():
        want, most = out[name].cpu().reshape(v.shape), bounds[name].cpu().reshape(v.shape)
        if name == "dx":
            most = most + half_step(dtype) * want.abs()
        off = (v.double() - want).abs()
        assert bool((off <= 1.01 * most + 1e-37).all()), (name, float((off / (most + 1e-37)).max()))


@pytest.mark.gpu
@pytest.mark.parametrize("bias", [False, True])
@pytest.mark.parametrize("dtype", [vcnn.F32, vcnn.BF16])
@pytest.mark.parametrize("batch,in_f,classes", SHAPES + LARGE)
def test_cost_and_gradients(batch, in_f, classes, dtype, bias):
    x, w, b, labels = inputs(batch, in_f, classes, dtype)
    b = b if bias else None
    ref = plain(x, w, b, labels)
    got = run(dtype, x, w, b, labels)
    check(dtype, got, *ref)
    alone = run(dtype, x, w, b, labels, want="each")
    check(dtype, alone, *ref)
    again = run(dtype, x, w, b, labels)
    assert all(torch.equal(got[n], again[n]) for n in got)


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [vcnn.F32, vcnn.BF16])
@pytest.mark.parametrize("batch,in_f,classes", [(300, 129, 700), (200, 64, 10), (1000, 256, 2049)])
def test_parts_offsets_and_single_outputs(batch, in_f, classes, dtype):
    x, w, b, labels = inputs(batch, in_f, classes, dtype, seed=2)
    ref = plain(x, w, b, labels)
    for part in (64, 130):
        check(dtype, run(dtype, x, w, b, labels, part=part, offset=1), *ref)
    check(dtype, run(dtype, x, w, b, labels, part=64, want="each"), *ref)
    for name in ("dx", "dw", "db"):  # (small float layers add dbias inside dw's product, or, alone, by itself: other roundings)
        check(dtype, run(dtype, x, w, b, labels, want=name), *ref)
    assert torch.equal(run(dtype, x, w, b, labels, want="")["loss"], run(dtype, x, w, b, labels, want="each")["loss"])


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [vcnn.F32, vcnn.BF16])
@pytest.mark.parametrize("batch,in_f,classes", [(40, 72, 300), (300, 72, 3000)])
def test_ignored_samples_and_impossible_classes(batch, in_f, classes, dtype):
    x, w, b, labels = inputs(batch, in_f, classes, dtype, ignored=0.5, seed=3)
    b[torch.arange(0, classes, 3)] = float("-inf")
    b[: min(200, classes // 2)] = float("-inf")  # whole tiles of them
    free = torch.nonzero(torch.isfinite(b))[:, 0]
    counted = labels != IGNORE
    labels[counted] = free[labels[counted].long() % len(free)].to(torch.int32)
    clean = run(dtype, x, w, b, labels)
    for fill in (float("nan"), float("inf"), 3e38):  # whatever ignored samples hold
        x[~counted] = fill
        got = run(dtype, x, w, b, labels)
        assert all(torch.equal(got[n], clean[n]) for n in got)
        assert torch.equal(run(dtype, x, w, b, labels, want="each")["each"] == 0, ~counted | (clean["each"] == 0))
    assert bool((clean["dx"][~counted] == 0).all()) and bool((clean["each"][~counted] == 0).all())
    masked = ~torch.isfinite(b)
    assert bool((clean["dw"][masked] == 0).all()) and bool((clean["db"][masked] == 0).all())
    keep = torch.nonzero(~masked)[:, 0]
    index = torch.full((classes,), -1, dtype=torch.int32)
    index[keep] = torch.arange(len(keep), dtype=torch.int32)
    fewer = torch.where(counted, index[labels.clamp(min=0).long()], labels)
    x[~counted] = 0.0
    ref = plain(x, w[keep], b[keep], fewer)
    check(dtype, {n: (v[keep] if n in ("dw", "db") else v) for n, v in clean.items()}, *ref)
    # nothing counts
    none = run(dtype, x, w, b, torch.full_like(labels, IGNORE))
    assert all(bool((v == 0).all()) for v in none.values())
    # the only label is impossible
    labels[:] = IGNORE
    labels[1] = int(torch.nonzero(masked)[0])
    got = run(dtype, x, w, b, labels)
    assert float(got["loss"]) == float("inf") and float(got["each"][1]) == float("inf")
    assert bool(torch.isfinite(got["dx"]).all()) and float(got["db"][labels[1].long()]) == -1.0


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [vcnn.F32, vcnn.BF16])
@pytest.mark.parametrize("bad", [-1, 300, 2 ** 31 - 1, -2 ** 31])
def test_bad_labels_and_values_show(dtype, bad):
    batch, in_f, classes = 70, 40, 300
    x, w, b, labels = inputs(batch, in_f, classes, dtype, seed=4)
    fine = run(dtype, x, w, b, labels)
    labels[5] = bad
    got = run(dtype, x, w, b, labels)
    others = torch.arange(batch) != 5
    assert bool(torch.isnan(got["loss"]).all()) and bool(torch.isnan(got["each"][5])) and bool(torch.isnan(got["dx"][5]).all())
    assert torch.equal(got["each"][others], fine["each"][others]) and bool(torch.isfinite(got["dx"][others]).all())
    assert bool(torch.isnan(got["dw"]).all()) and bool(torch.isnan(got["db"]).all())
    for value in (float("nan"), float("inf")):
        y = x.clone()
        labels[5] = 7
        y[5, 3] = value
        got = run(dtype, y, w, b, labels)
        assert bool(torch.isnan(got["each"][5])) and bool(torch.isnan(got["dx"][5]).any())
        assert torch.equal(got["each"][others], fine["each"][others])


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [vcnn.F32, vcnn.BF16])
def test_logits_far_from_zero(dtype):
    """Logits of thousands of either sign: nothing overflows, and the cost is their distance."""
    batch, in_f, classes = 33, 16, 500
    x, w, b, labels = inputs(batch, in_f, classes, dtype, ignored=0.0, seed=5)
    b = b * 1e4
    ref = plain(x, w, b, labels)
    check(dtype, run(dtype, x, w, b, labels), *ref)
    ref = plain((x.float() * 1e3).to(x.dtype), w, None, labels)
    check(dtype, run(dtype, (x.float() * 1e3).to(x.dtype), w, None, labels), *ref)


@pytest.mark.gpu
@pytest.mark.parametrize("batch,in_f,classes", [(6, 20, 33), (150, 24, 400)])
def test_gradients_against_differences(batch, in_f, classes):
    """The cost along a direction of x, w and bias: values of the formula in 64 bits on both sides, and the float gradients."""
    x, w, b, labels = inputs(batch, in_f, classes, vcnn.F32, seed=6)
    got = run(vcnn.F32, x, w, b, labels)
    out, bounds, gradients = plain(x, w, b, labels)
    gradients(0.0, 0.0)
    g, e = torch.Generator().manual_seed(7), 1e-5
    ways = [torch.randn(t.shape, generator=g, dtype=torch.float64) for t in (x, w, b)]

    def cost(s):
        return float(plain(*(t.double() + s * way for t, way in zip((x, w, b), ways)), labels)[0]["loss"])

    slope = (cost(e) - cost(-e)) / (2 * e)
    ours = sum(float((got[n].double() * way).sum()) for n, way in zip(("dx", "dw", "db"), ways))
    slack = sum(float((bounds[n].cpu() * way.abs()).sum()) for n, way in zip(("dx", "dw", "db"), ways))
    assert abs(ours - slope) <= 1.01 * slack + 1e-6 * abs(slope) + 1e-7  # e^2 times a third derivative of the order of 10^2 slopes


@pytest.mark.gpu
@pytest.mark.parametrize("batch,in_f,classes", [(200, 136, 1100), (300, 520, 1100), (12, 100, 700), (128, 50, 10)])
@pytest.mark.parametrize("dtype", [vcnn.F32, vcnn.BF16])
def test_captured_call(batch, in_f, classes, dtype):
    """Replayed on new inputs, with eager calls on a workspace of their own between the replays."""
    x, w, b, labels = (dev(t) for t in inputs(batch, in_f, classes, dtype, seed=8))
    nbytes = vcnn.fc_softmax_loss_workspace_bytes(dtype, batch, in_f, classes, True)

    def buffers():
        return dict(loss=torch.zeros((), device=DEV), each=torch.zeros(batch, device=DEV), dx=torch.zeros_like(x),
                    dw=torch.zeros(classes, in_f, device=DEV), db=torch.zeros(classes, device=DEV),
                    ws=torch.empty(nbytes, dtype=torch.uint8, device=DEV))

    def call(o):
        vcnn.fc_softmax_loss(dtype, batch, in_f, classes, x, w, b, labels, IGNORE, o["loss"], o["each"], o["dx"], o["dw"], o["db"],
                             o["ws"])

    o, eager = buffers(), buffers()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        call(o)
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call(o)
    for n in range(4):
        nx, _, _, nl = inputs(batch, in_f, classes, dtype, seed=20 + n)
        x.copy_(dev(nx)), labels.copy_(dev(nl))
        call(eager)
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(o[k], eager[k]) for k in ("loss", "each", "dx", "dw", "db"))


@pytest.mark.gpu
@pytest.mark.parametrize("scale", [1e-30, 1e-20, 1e15, 1e30])
@pytest.mark.parametrize("batch", [12, 300])
def test_float_operands_of_any_magnitude(batch, scale):
    """x and w far from one, their products ordinary; some rows of either much smaller than the others, one class of zeros."""
    in_f, classes = 520, 1100
    x, w, b, labels = inputs(batch, in_f, classes, vcnn.F32, seed=9)
    x, w = x * scale, w / scale
    x[1::3] *= 2.0 ** -6
    w[2::5] *= 2.0 ** -6
    w[7] = 0.0
    out, bounds, gradients = plain(x, w, b, labels)
    got = run(vcnn.F32, x, w, b, labels)
    check(vcnn.F32, got, out, bounds, gradients)


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [vcnn.F32, vcnn.BF16])
def test_one_sample_apart_does_not_move_the_others(dtype):
    """A sample of 2^20 times the others' magnitude, in the products that scale all of x together: the others' costs stay within
    what 2^-39 of the largest element leaves in their logits."""
    batch, in_f, classes = 300, 520, 1100
    x, w, b, labels = inputs(batch, in_f, classes, dtype, ignored=0.0, seed=10)
    x[5] = (x[5].float() * 2.0 ** 20).to(x.dtype)
    out, bounds, _ = plain(x, w, b, labels)
    got = run(dtype, x, w, b, labels, want="each")["each"].double()
    lost = 2 * 2.0 ** -39 * float(x.float().abs().max()) * w.float().abs().sum(1).max().double() * (dtype == vcnn.F32)
    others = torch.arange(batch) != 5
    assert bool(((got - out["each"].cpu()).abs() <= 1.01 * bounds["each"].cpu() + lost)[others].all())


@pytest.mark.gpu
def test_weights_of_more_than_2_31_elements():
    """Rows behind 2^32 bytes, read where they stand by the kernels for few samples and by those for many."""
    in_f, classes = 20480, 110000
    free, _ = torch.cuda.mem_get_info()
    if free < 24 << 30:
        pytest.skip("needs 24 GiB")
    g = torch.Generator(device=DEV).manual_seed(11)
    w = torch.empty(classes, in_f, dtype=torch.bfloat16, device=DEV)
    for at in range(0, classes, 10000):
        w[at:at + 10000] = torch.randn(min(10000, classes - at), in_f, device=DEV, generator=g).bfloat16() / 64
    for batch in (3, 70):
        labels = torch.randint(0, classes, (batch,), dtype=torch.int32, device=DEV, generator=g)
        labels[0] = classes - 1
        x = (torch.randn(batch, in_f, device=DEV, generator=g) + 20 * w[labels.long()].float()).bfloat16()
        z = torch.cat([x.float() @ w[at:at + 10000].float().t().contiguous() for at in range(0, classes, 10000)], 1).double()
        want = torch.logsumexp(z, 1) - z.gather(1, labels.long()[:, None])[:, 0]
        loss, each = torch.empty((), device=DEV), torch.empty(batch, device=DEV)
        ws = torch.empty(vcnn.fc_softmax_loss_workspace_bytes(vcnn.BF16, batch, in_f, classes, False), dtype=torch.uint8, device=DEV)
        vcnn.fc_softmax_loss(vcnn.BF16, batch, in_f, classes, x, w, None, labels, IGNORE, loss, each, None, None, None, ws)
        # both sides' sums: at most in_f roundings of the sum of magnitudes each, here some 20 * in_f / 64 / 64 + 2 |x| |w|
        most = 2 * 2 * (in_f / 16) * U * float((x.float().abs() @ w[:1000].float().abs().t()).max()) * 2
        assert float((each.double() - want).abs().max()) <= most


def test_refusals_need_no_gpu():
    lib, f = vcnn.lib(), 0x1000  # never dereferenced: validation fails first

    def call(dtype=vcnn.BF16, batch=4, in_f=16, classes=10, x=f, w=f, labels=f, loss=f, dx=None, ws=f, nbytes=1 << 30):
        return lib.vcnn_fc_softmax_loss(dtype, batch, in_f, classes, x, w, None, labels, -1, loss, None, dx, None, None, ws, nbytes, None)

    for name in ("batch", "in_f", "classes"):
        assert call(**{name: 0}) == vcnn.ERR_SHAPE and call(**{name: -3}) == vcnn.ERR_SHAPE
    assert call(dtype=7) == vcnn.ERR_UNSUPPORTED
    assert call(in_f=(1 << 22) + 1) == vcnn.ERR_UNSUPPORTED and call(classes=(1 << 22) + 1) == vcnn.ERR_UNSUPPORTED
    assert call(in_f=1 << 20, classes=1 << 20) == vcnn.ERR_UNSUPPORTED
    for name in ("x", "w", "labels", "loss"):
        assert call(**{name: None}) == vcnn.ERR_NULL
    assert call(w=0x1008) == vcnn.ERR_UNSUPPORTED  # rows of bfloat16 that are read where they stand
    for dtype in (vcnn.F32, vcnn.BF16):
        need = vcnn.fc_softmax_loss_workspace_bytes(dtype, 4, 16, 10, True)
        assert need >= vcnn.fc_softmax_loss_workspace_bytes(dtype, 4, 16, 10, False) > 0
        assert call(dtype=dtype, dx=f, ws=None) == vcnn.ERR_WORKSPACE
        assert call(dtype=dtype, dx=f, ws=0x1010) == vcnn.ERR_WORKSPACE
        assert call(dtype=dtype, dx=f, ws=0x1100, nbytes=need - 256) == vcnn.ERR_WORKSPACE
        # room for the logits of a part, whatever the batch
        large = vcnn.fc_softmax_loss_workspace_bytes(dtype, 1 << 20, 64, 100000, True)
        assert large < (1 << 30) + (1 << 28)
    with pytest.raises(vcnn.VcnnError):
        vcnn.fc_softmax_loss_workspace_bytes(vcnn.F32, 0, 1, 1, False)
    assert lib.vcnn_fc_softmax_loss_workspace_bytes(vcnn.F32, 1, 1, 1, 0, None) == vcnn.ERR_NULL
