"""A network with norms, trained with Muon through TrainStep, against the same in 64 bits (torch's autograd on the CPU), and
its fully connected end answering in 8 bits."""
import numpy as np
import pytest
import torch
import torch.nn.functional as F

from paper_1501_07338_amd import vcnn
from paper_1501_07338_amd import workloads as wl
from paper_1501_07338_amd.net import TrainStep
from test_gpu_muon import products
from util import TOL_F32, rel_err

MUON = dict(lr=0.03, momentum=0.9, nesterov=True, weight_decay=0.05, steps=5)


def normed(batch=24):
    return wl.Net("normed", 9, batch, (1, 14, 14),
                  [wl.Conv(8, 3, 3, relu=True), wl.Pool(2, 2), wl.Norm(), wl.FC(40, relu=True), wl.Norm(), wl.FC(10)],
                  "softmax", classes=10, lr=0.02)


def inputs_of(net):
    rng = np.random.Generator(np.random.Philox(key=90))
    return dict(x=rng.random((net.batch,) + net.in_chw).astype(np.float32),
                labels=rng.integers(0, 10, net.batch).astype(np.int32))


def forward64(net, params, x):
    a = x
    for L, p in zip(net.layers, params):
        if isinstance(L, wl.Pool):
            a = F.max_pool2d(a, L.win, L.stride)
        elif isinstance(L, wl.Norm):
            flat = a.reshape(a.shape[0], -1)
            a = (flat * (flat.square().mean(1, keepdim=True) + L.eps).rsqrt() * p[0]).reshape(a.shape)
        else:
            a = F.conv2d(a, *p) if isinstance(L, wl.Conv) else F.linear(a.reshape(a.shape[0], -1), *p)
            a = a.relu() if L.relu else a
    return a


def test_shapes_and_parameters():
    net = normed()
    assert net.shapes == [(24, 8, 12, 12), (24, 8, 6, 6), (24, 8, 6, 6), (24, 40), (24, 40), (24, 10)]
    p = wl.make_params(net)
    assert p[1] is None and p[2][0].shape == (288,) and p[4][0].shape == (40,) and len(p[2]) == 1
    assert np.all(p[2][0] == 1.0) and p[3][0].shape == (40, 288)


@pytest.mark.gpu
@pytest.mark.parametrize("captured", [False, True])
def test_steps_against_64_bits(captured):
    net, lr = normed(), MUON["lr"]
    inputs, params = inputs_of(net), wl.make_params(net)
    ts = TrainStep(net, params, inputs, first_layer_dx=True, muon=MUON)
    ps = [None if p is None else [torch.from_numpy(t).double() for t in p] for p in params]
    ms = [None if p is None or len(p) == 1 else torch.zeros_like(p[0]) for p in ps]
    x, labels = torch.from_numpy(inputs["x"]).double(), torch.from_numpy(inputs["labels"]).long()
    if captured:
        ts.snapshot()
        graph = ts.capture()  # (runs a step by itself)
        torch.cuda.synchronize()
        ts.restore()
    for _ in range(3):
        for p in ps:
            for t in p or ():
                t.requires_grad_(True)
        loss = F.cross_entropy(forward64(net, ps, x), labels)
        grads = torch.autograd.grad(loss, [t for p in ps for t in p or ()])
        if captured:
            graph.replay()
        else:
            ts.step()
        torch.cuda.synchronize()
        assert abs(float(ts.loss) - float(loss.detach())) <= TOL_F32 * float(loss.detach())
        got = [t for g in ts.grads if g is not None for t in g]
        for a, b in zip(got, grads):
            assert rel_err(a.cpu().numpy(), b.numpy()) <= TOL_F32
        it = iter(grads)
        for li, p in enumerate(ps):
            if p is None:
                continue
            g = [next(it) for _ in p]
            p = [t.detach() for t in p]
            if len(p) == 2:
                rows = p[0].shape[0]
                ms[li] = MUON["momentum"] * ms[li] + g[0]
                o = products((g[0] + MUON["momentum"] * ms[li]).reshape(rows, -1), 5)
                scale = max(1.0, o.shape[0] / o.shape[1]) ** 0.5
                p[0] = (1 - lr * MUON["weight_decay"]) * p[0] - lr * scale * o.reshape(p[0].shape)
            p[-1] = p[-1] - net.lr * g[-1]
            ps[li] = p
    # (a gradient's error, TOL_F32 at most, is a perturbation of what is orthogonalised; the map's slope is at most 4^5 over its
    # five steps for directions that are nearly absent, and some 1 for the others: held to 20 times it)
    for a, b in zip(ts.params, ps):
        for t, u in zip(a or (), b or ()):
            assert rel_err(t.cpu().numpy(), u.detach().numpy()) <= 20 * TOL_F32


@pytest.mark.gpu
def test_bf16_chain_and_its_working_copies():
    net = normed()
    ts = TrainStep(net, wl.make_params(net), inputs_of(net), dtype=vcnn.BF16, muon=dict(lr=0.01))
    for _ in range(2):
        ts.step()
    torch.cuda.synchronize()
    assert bool(torch.isfinite(ts.loss))
    for li in (2, 4):  # a norm's output from the input that it stored, half a step of bfloat16 off
        h = ts.acts[li].double().flatten(1)
        gain = ts.params[li][0].double() + net.lr * ts.grads[li][0].double()  # as the forward pass had it
        want = h * (h.square().mean(1, keepdim=True) + net.layers[li].eps).rsqrt() * gain
        got = ts.acts[li + 1].double().flatten(1)
        assert bool(((got - want).abs() <= want.abs() * (2.0 ** -8 + 1e-5)).all())
    for p, h in zip(ts.params, ts.params16):
        if h is not None:
            assert torch.equal(p[0].to(torch.bfloat16), h)


@pytest.mark.gpu
def test_trained_then_answered_in_eight_bits():
    """Trains a few steps, quantises the weights once, and answers from the trunk's features by norm and 8-bit product."""
    net = normed()
    inputs, params = inputs_of(net), wl.make_params(net)
    ts = TrainStep(net, params, inputs, muon=MUON)
    for _ in range(3):
        ts.step()
    ts.forward()
    (w, b), gain = ts.params[3], ts.params[2][0]
    rows, cols = 24, 288
    wq, ws = torch.empty(40, cols, dtype=torch.int8, device=w.device), torch.empty(40, device=w.device)
    q, s = torch.empty(rows, cols, dtype=torch.int8, device=w.device), torch.empty(rows, device=w.device)
    y = torch.empty(rows, 40, device=w.device)
    vcnn.quant_rows_i8(vcnn.F32, 40, cols, w, wq, ws)
    vcnn.rmsnorm_fwd_i8(vcnn.F32, rows, cols, net.layers[2].eps, ts.acts[2], None, gain, None, q, s)
    vcnn.fc_fwd_i8(vcnn.F32, rows, cols, 40, vcnn.ACT_RELU, q, s, wq, ws, b, y)
    torch.cuda.synchronize()
    # each operand is off by half a step an element (see the 8-bit layer's tests)
    z, dz, dw = ts.acts[3].reshape(rows, cols), s[:, None] / 2, ws[None, :] / 2
    bound = z.abs().sum(1, keepdim=True) * dw + w.abs().sum(1)[None, :] * dz + cols * dz * dw
    assert bool(((y - ts.acts[4]).abs() <= bound * 1.001 + 1e-6).all())


def test_unknown_settings_are_refused():
    with pytest.raises(ValueError, match="Muon"):
        dummy = TrainStep.__new__(TrainStep)
        net = normed()
        dummy.__init__(net, wl.make_params(net), inputs_of(net), device="cpu", overlap=False, muon=dict(rate=1.0))
