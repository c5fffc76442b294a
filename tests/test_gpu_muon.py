"""Orthogonalisation by Newton-Schulz products and the Muon update against the same in 64 bits.

Tolerances.  A step perturbs every factor of a X + b A X + c A^2 X (one, three, five factors of X or of what is made of
them) by at most 2^-23 of itself, and the sums by no more: (a + 3 |b| + 5 c) 2^-23 = 28 * 2^-23 of |X|.  The map's slope is
at most 4 on [0, 1.21], so `steps` steps add up to at most 28 * 2^-23 * (4^steps - 1) / 3 of the largest norm on the
way, sqrt(small side) * 1.21.  That is a worst case; a matrix of ordinary size is also held to twice the error that the
same products in float arithmetic have: an operand of two f16 terms is off by up to 2^-23 where a float is by 2^-24, and
the sums are rounded no more often."""
import ctypes

import pytest
import torch

from paper_1501_07338_amd import vcnn
from test_gpu_norm import DEV, Guarded, dev

A, B, C = 3.4445, -4.7750, 2.0315
U = 2.0 ** -24
SHAPES = [(1, 1), (1, 9), (7, 1), (3, 5), (20, 25), (64, 800), (500, 50), (127, 129), (128, 128), (129, 260), (300, 1000),
          (513, 40), (700, 650), (60, 5000), (4100, 130), (200, 9000)]


def matrix(seed, rows, cols):
    """A few strong directions over a full-rank rest."""
    g = torch.Generator().manual_seed(seed)
    k = max(1, min(rows, cols) // 16)
    return 1e-3 * (torch.randn(rows, k, generator=g) @ torch.randn(k, cols, generator=g) + torch.randn(rows, cols, generator=g))


def products(g, steps):
    """The definition, in g's type; on the smaller side."""
    x = g.t() if g.shape[0] > g.shape[1] else g
    norm = torch.linalg.vector_norm(x.double()).to(x.dtype)
    x = x / norm if float(norm) > 0 else x * 0
    for _ in range(steps):
        a = x @ x.t()
        x = A * x + (B * a + C * (a @ a)) @ x
    return x.t() if g.shape[0] > g.shape[1] else x


def bound(rows, cols, steps):
    return 28 * 2.0 ** -23 * (4 ** steps - 1) / 3 * 1.21 * min(rows, cols) ** 0.5


def workspace(n):
    return torch.empty(max(n, 256), dtype=torch.uint8, device=DEV)


def orthogonal(g, steps=5):
    rows, cols = g.shape
    out = Guarded((rows, cols), torch.float32)
    vcnn.orthogonalize(rows, cols, steps, dev(g), out.t, workspace(vcnn.orthogonalize_workspace_bytes(rows, cols)))
    return out.cpu()


@pytest.mark.gpu
@pytest.mark.parametrize("steps", [1, 2, 5])
@pytest.mark.parametrize("rows,cols", SHAPES)
def test_against_64_bits(rows, cols, steps):
    g = matrix(rows + cols, rows, cols)
    want = products(g.double(), steps)
    got = orthogonal(g, steps).double()
    off = float(torch.linalg.vector_norm(got - want))
    assert off <= bound(rows, cols, steps)
    if min(rows, cols) >= 64:
        assert off <= 2 * float(torch.linalg.vector_norm(products(g, steps).double() - want))


def large(seed, rows, cols):
    g = torch.Generator(device=DEV).manual_seed(seed)
    k = min(rows, cols) // 16
    return torch.randn(rows, k, device=DEV, generator=g) @ torch.randn(k, cols, device=DEV, generator=g) + \
        torch.randn(rows, cols, device=DEV, generator=g)


@pytest.mark.gpu
@pytest.mark.parametrize("rows,cols", [(1500, 1570), (2150, 2070), (2900, 2950), (4000, 4100), (5900, 5830)])
def test_every_tile(rows, cols):
    """Sizes at which the phases take the larger tiles, one kind after the other."""
    g = large(rows, rows, cols)
    out = Guarded((rows, cols), torch.float32)
    vcnn.orthogonalize(rows, cols, 3, g, out.t, workspace(vcnn.orthogonalize_workspace_bytes(rows, cols)))
    out.cpu()
    want = products(g.double(), 3)
    off = float(torch.linalg.vector_norm(out.t.double() - want))
    assert off <= bound(rows, cols, 3)
    assert off <= 2 * float(torch.linalg.vector_norm(products(g, 3).double() - want))


@pytest.mark.gpu
@pytest.mark.parametrize("shapes", [[(300, 5000), (2150, 1300), (1200, 4100), (7, 9)], [(40, 9000), (6000, 70), (130, 2100)]],
                         ids=["large", "long sums"])
def test_update_of_unlike_matrices(shapes):
    lr, mu = 0.05, 0.9
    ms, dws = [large(i, *s) for i, s in enumerate(shapes)], [large(9 + i, *s) for i, s in enumerate(shapes)]
    ws = [torch.zeros(s, device=DEV) for s in shapes]
    kept = [m.clone() for m in ms]
    vcnn.muon_update_multi(lr, mu, True, 0.0, 5, ws, dws, ms, workspace(vcnn.muon_workspace_bytes(shapes)))
    for (rows, cols), w, g, m in zip(shapes, ws, dws, kept):
        u = g.double() + mu * (mu * m.double() + g.double())
        step = lr * max(1.0, rows / cols) ** 0.5
        want = -step * products(u, 5)
        off = float(torch.linalg.vector_norm(w.double() - want))
        assert off <= step * 2 * bound(rows, cols, 5)  # (u as floats: as above)
        if min(rows, cols) >= 64:
            f = step * float(torch.linalg.vector_norm(products(u.float(), 5).double() - want / -step))
            assert off <= 2 * f + 4 * U * float(torch.linalg.vector_norm(want))


@pytest.mark.gpu
def test_singular_values_come_near_one():
    g = torch.linalg.qr(torch.randn(200, 200, generator=torch.Generator().manual_seed(1), dtype=torch.float64))[0]
    s = torch.logspace(0, -1, 200, dtype=torch.float64)  # the norm is some 5.5: down to 0.018 of it
    h = torch.linalg.qr(torch.randn(330, 200, generator=torch.Generator().manual_seed(2), dtype=torch.float64))[0]
    m = (g * s) @ h.t()
    out = orthogonal(m.float()).double()
    assert 0.67 <= float(torch.linalg.svdvals(out).min()) and float(torch.linalg.svdvals(out).max()) <= 1.21
    # the singular vectors stay: in their bases the result is diagonal
    d = g.t() @ out @ h
    assert float((d - torch.diag(torch.diag(d))).abs().max()) <= bound(200, 330, 5)


@pytest.mark.gpu
@pytest.mark.parametrize("rows,cols", [(40, 70), (300, 130)])
def test_ranges(rows, cols):
    g = matrix(3, rows, cols)
    plain = orthogonal(g)
    for e in (100, -60):  # powers of two leave the bits (the squares of the first leave the float range)
        assert torch.equal(orthogonal(g * 2.0 ** e), plain)
    assert torch.equal(orthogonal(torch.zeros(rows, cols)), torch.zeros(rows, cols))
    one = torch.zeros(rows, cols)
    one[rows - 1, cols - 1] = -3.0  # a single entry: the scalar map
    v = 1.0
    for _ in range(5):
        v = A * v + B * v ** 3 + C * v ** 5
    got = orthogonal(one)
    assert abs(float(got[rows - 1, cols - 1]) + v) <= bound(1, 1, 5) and int((got != 0).sum()) == 1
    for bad in (float("inf"), float("-inf"), float("nan")):
        h = g.clone()
        h[0, cols // 2] = bad
        assert bool(torch.isnan(orthogonal(h)).all())
    low = torch.randn(rows, 3, generator=torch.Generator().manual_seed(4)) @ torch.randn(3, cols, generator=torch.Generator().manual_seed(5))
    off = float(torch.linalg.vector_norm(orthogonal(low).double() - products(low.double(), 5)))  # rank three
    assert off <= bound(rows, cols, 5)


@pytest.mark.gpu
def test_in_place():
    g = matrix(6, 90, 210)
    d = dev(g)
    vcnn.orthogonalize(90, 210, 5, d, d, workspace(vcnn.orthogonalize_workspace_bytes(90, 210)))
    assert torch.equal(d.cpu(), orthogonal(g))


def tensors(shapes, seed=0):
    w, dw, m = [], [], []
    for i, s in enumerate(shapes):
        rows, cols = s[0], int(torch.tensor(s[1:]).prod())
        w.append(torch.randn(s, generator=torch.Generator().manual_seed(seed + 3 * i)))
        dw.append(matrix(seed + 3 * i + 1, rows, cols).view(s))
        m.append(10 * matrix(seed + 3 * i + 2, rows, cols).view(s))
    return w, dw, m


DIGITS = [(20, 1, 5, 5), (50, 20, 5, 5), (500, 800), (10, 500)]


@pytest.mark.gpu
@pytest.mark.parametrize("nesterov", [False, True])
@pytest.mark.parametrize("shapes", [DIGITS, [(3, 7)] * 9 + [(40, 30)] * 6 + [(200, 100), (5, 2, 3, 3)] + [(64, 65)] * 5,
                                    [(3, 7), (40, 30), (64, 65), (500, 20), (5, 3000), (1, 1), (64, 64)]],
                         ids=["digits", "more than a batch", "small"])
def test_update(shapes, nesterov):
    lr, mu, decay = 0.05, 0.9, 0.1
    w, dw, m = tensors(shapes)
    wd, gd, md = ([dev(t) for t in ts] for ts in (w, dw, m))
    halves = [Guarded(s, torch.bfloat16) if i % 2 == 0 else None for i, s in enumerate(shapes)]
    vcnn.muon_update_multi(lr, mu, nesterov, decay, 5, wd, gd, md, workspace(vcnn.muon_workspace_bytes(shapes)),
                           [None if h is None else h.t for h in halves])
    torch.cuda.synchronize()
    for i, s in enumerate(shapes):
        rows, cols = s[0], w[i].numel() // s[0]
        mm = mu * m[i].double() + dw[i].double()
        assert bool(((md[i].cpu().double() - mm).abs() <= (mu * m[i].abs() + dw[i].abs()).double() * 3 * U).all())
        u = (dw[i].double() + mu * mm if nesterov else mm).view(rows, cols)
        step = lr * max(1.0, rows / cols) ** 0.5
        o = products(u, 5).view(s)
        want = (1 - lr * decay) * w[i].double() - step * o
        got = wd[i].cpu().double()
        # u, as floats, is off by 3 * 2^-24 of its terms (|u| is no smaller than a few tenths of them): as a perturbation of
        # X it grows as the others do
        off = step * 2 * bound(rows, cols, 5) + 4 * U * float(w[i].double().abs().max() + step)
        assert float((got - want).abs().max()) <= off
        if min(rows, cols) >= 40:  # tight: the direction by itself, from the update
            d = torch.linalg.vector_norm(got - want)
            f = step * torch.linalg.vector_norm(products(u.float(), 5).double().view(s) - o)
            assert float(d) <= 2 * float(f) + 4 * U * float(torch.linalg.vector_norm(w[i].double().abs() + step * o.abs()))
        if halves[i] is not None:
            assert torch.equal(halves[i].cpu(), wd[i].cpu().to(torch.bfloat16))
        assert torch.equal(gd[i].cpu(), dw[i])


@pytest.mark.gpu
@pytest.mark.parametrize("shapes", [DIGITS, DIGITS[:2], [(300, 5000), (70, 2100)]], ids=["digits", "small", "shared sums"])
def test_the_same_bits_in_every_run_and_replayed(shapes):
    """Eager calls, calls on a stream of their own and a graph's replays give the same bits, step after step."""
    w, dw, m = tensors(shapes, 50)

    def fresh():
        return [[dev(t) for t in ts] for ts in (w, dw, m)]

    def go(ts, ws):
        vcnn.muon_update_multi(0.02, 0.95, True, 0.0, 5, *ts, ws)

    ws = workspace(vcnn.muon_workspace_bytes(shapes))
    eager, other, replayed = fresh(), fresh(), fresh()
    for _ in range(3):
        go(eager, ws)
        ws.fill_(255)  # nothing is carried from call to call in the workspace
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        for _ in range(3):
            go(other, ws)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        go(replayed, ws)
    for _ in range(3):
        graph.replay()
        torch.cuda.synchronize()
        ws.fill_(255)
    torch.cuda.synchronize()
    for a, b, c in zip(eager[0] + eager[2], other[0] + other[2], replayed[0] + replayed[2]):
        assert torch.equal(a, b) and torch.equal(a, c)


def test_refusals_need_no_gpu():
    lib = vcnn.lib()
    f, need = 0x1000, ctypes.c_size_t()
    for rows, cols, st in ((0, 4, vcnn.ERR_SHAPE), (4, -1, vcnn.ERR_SHAPE), ((1 << 24) + 1, 1, vcnn.ERR_UNSUPPORTED),
                           (1 << 20, 1 << 20, vcnn.ERR_UNSUPPORTED)):
        assert lib.vcnn_orthogonalize_workspace_bytes(rows, cols, ctypes.byref(need)) == st
        assert lib.vcnn_orthogonalize(rows, cols, 5, f, f, f, 1 << 60, None) == st
    n = vcnn.orthogonalize_workspace_bytes(4, 8)
    for steps in (0, -1, 33):
        assert lib.vcnn_orthogonalize(4, 8, steps, f, f, 0x1000, n, None) == vcnn.ERR_UNSUPPORTED
    assert lib.vcnn_orthogonalize(4, 8, 5, None, f, 0x1000, n, None) == vcnn.ERR_NULL
    assert lib.vcnn_orthogonalize(4, 8, 5, f, None, 0x1000, n, None) == vcnn.ERR_NULL
    for ws, size in ((None, 0), (0x1010, n), (0x1000, n - 1)):
        assert lib.vcnn_orthogonalize(4, 8, 5, f, f, ws, size, None) == vcnn.ERR_WORKSPACE
    assert lib.vcnn_orthogonalize_workspace_bytes(4, 8, None) == vcnn.ERR_NULL
    assert n == vcnn.muon_workspace_bytes([(4, 8)]) and vcnn.muon_workspace_bytes([]) == 0
    sixteen = vcnn.muon_workspace_bytes([(4, 8)] * 16)
    assert n < sixteen < 16 * n and sixteen == vcnn.muon_workspace_bytes([(4, 8)] * 40)  # (batches share it)

    def go(count=1, p=(f, f, f), lr=0.1, mu=0.9, wd=0.0, steps=5, ws=0x1000, size=n):
        one = (ctypes.c_int32 * 1)
        ptr = [None if v is None else (ctypes.c_void_p * 1)(v or None) for v in p]
        return lib.vcnn_muon_update_multi(count, one(4), one(8), *ptr, None, ctypes.c_float(lr), ctypes.c_float(mu), 1,
                                          ctypes.c_float(wd), steps, ws, size, None)

    assert go(count=-1) == vcnn.ERR_SHAPE and go(count=0, p=(None,) * 3, ws=None) == vcnn.OK
    assert go(steps=0) == vcnn.ERR_UNSUPPORTED
    for v in (float("nan"), float("inf")):
        assert go(lr=v) == go(mu=v) == go(wd=v) == vcnn.ERR_UNSUPPORTED
    for i in range(3):
        assert go(p=tuple(None if j == i else f for j in range(3))) == vcnn.ERR_NULL
        assert go(p=tuple(0 if j == i else f for j in range(3))) == vcnn.ERR_NULL
    assert go(ws=None, size=0) == go(ws=0x1010) == go(size=n - 1) == vcnn.ERR_WORKSPACE
    assert lib.vcnn_muon_update_multi(1, None, None, None, None, None, None, ctypes.c_float(0), ctypes.c_float(0), 0,
                                      ctypes.c_float(0), 5, None, 0, None) == vcnn.ERR_NULL
