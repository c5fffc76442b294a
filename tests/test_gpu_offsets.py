"""Tensors of more than 2^31 elements: the last rows of the norm, the 8-bit layer and the orthogonalisation."""
import pytest
import torch

from paper_1501_07338_amd import vcnn
from test_gpu_int8 import U, reference
from test_gpu_muon import A, B, C, bound
from test_gpu_norm import DEV, EPS, depth, half_step, integers

pytestmark = pytest.mark.gpu


def test_rows_behind_2_31_elements():
    rows, cols = 66_000, 33_000
    x = torch.zeros(rows, cols, dtype=torch.bfloat16, device=DEV)
    last = torch.randn(3, cols, device=DEV).to(torch.bfloat16)
    x[-3:] = last
    q, s = torch.empty(rows, cols, dtype=torch.int8, device=DEV), torch.empty(rows, device=DEV)
    vcnn.quant_rows_i8(vcnn.BF16, rows, cols, x, q, s)
    want, a = integers(last.float())
    assert torch.equal(q[-3:].double(), want) and bool(((s[-3:].double() - a / 127).abs() <= a / 127 * 2 * U).all())
    assert float(s[:-3].max()) == 0.0
    del q
    gain, rstd = torch.ones(cols, device=DEV), torch.empty(rows, device=DEV)
    y = torch.empty_like(x)
    vcnn.rmsnorm_fwd(vcnn.BF16, rows, cols, EPS, x, None, gain, None, y, rstd)
    r = (last.double().square().mean(1) + EPS).rsqrt()
    want = last.double() * r[:, None]
    assert bool(((y[-3:].double() - want).abs() <= want.abs() * (half_step(vcnn.BF16) + depth(cols) * U) * 1.01).all())
    dg = torch.empty(cols, device=DEV)
    ws = torch.empty(vcnn.rmsnorm_workspace_bytes(rows, cols), dtype=torch.uint8, device=DEV)
    dh = torch.empty_like(x)
    vcnn.rmsnorm_bwd(vcnn.BF16, rows, cols, x, gain, rstd, y, None, dh, dg, ws)  # dy = y: only the last rows count
    yd = y[-3:].double()
    z = last.double() * rstd[-3:].double()[:, None]
    want = rstd[-3:].double()[:, None] * (yd - z * (yd * z).mean(1, keepdim=True))
    size = rstd[-3:].double()[:, None] * (yd.abs() + z.abs() * (yd * z).abs().mean(1, keepdim=True))
    off = (dh[-3:].double() - want).abs()
    assert bool((off <= want.abs() * half_step(vcnn.BF16) * 1.01 + size * depth(cols) * U).all())
    want, size = (yd * z).sum(0), (yd * z).abs().sum(0)
    assert bool(((dg.double() - want).abs() <= size * (rows // 512 + 70) * U).all())


@pytest.mark.parametrize("batch", [1, 20, 130])
def test_weights_behind_2_31_bytes(batch):
    out, k = 17_000, 131_071
    w = torch.zeros(out, k, dtype=torch.int8, device=DEV)
    g = torch.Generator().manual_seed(batch)
    last = torch.randint(-127, 128, (40, k), generator=g, dtype=torch.int8)
    x = torch.randint(-127, 128, (batch, k), generator=g, dtype=torch.int8)
    w[-40:] = last.to(DEV)
    xs, ws = torch.rand(batch, generator=g) / 1e4, torch.rand(out, generator=g) / 1e4
    y = torch.empty(batch, out, device=DEV)
    work = torch.empty(max(256, vcnn.fc_i8_workspace_bytes(batch, k, out)), dtype=torch.uint8, device=DEV)
    vcnn.fc_fwd_i8(vcnn.F32, batch, k, out, vcnn.ACT_NONE, x.to(DEV), xs.to(DEV), w, ws.to(DEV), None, y, work)
    want, size = reference(x, last, xs, ws[-40:], None, vcnn.ACT_NONE)
    got = y.cpu().double()
    assert bool(((got[:, -40:] - want).abs() <= size * 5 * U).all()) and float(got[:, :-40].abs().max()) == 0.0


def test_outputs_behind_2_31_elements():
    batch, out, k = 70_000, 33_000, 64
    g = torch.Generator().manual_seed(1)
    x = torch.randint(-127, 128, (batch, k), generator=g, dtype=torch.int8)
    w = torch.randint(-127, 128, (out, k), generator=g, dtype=torch.int8)
    xs, ws = torch.rand(batch, generator=g) / 1e2, torch.rand(out, generator=g) / 1e2
    y = torch.empty(batch, out, dtype=torch.bfloat16, device=DEV)
    vcnn.fc_fwd_i8(vcnn.BF16, batch, k, out, vcnn.ACT_NONE, x.to(DEV), xs.to(DEV), w.to(DEV), ws.to(DEV), None, y)
    want, size = reference(x[-5:], w, xs[-5:], ws, None, vcnn.ACT_NONE)
    off = (y[-5:].cpu().double() - want).abs()
    assert bool((off <= want.abs() * half_step(vcnn.BF16) * 1.01 + size * 4 * U).all())


@pytest.mark.parametrize("tall", [False, True])
def test_matrices_behind_2_31_elements(tall):
    small, large = 130, 1 << 24
    shape = (large, small) if tall else (small, large)
    gen = torch.Generator(device=DEV).manual_seed(2)
    g = torch.randn(*shape, device=DEV, generator=gen)
    out = torch.empty_like(g)
    ws = torch.empty(vcnn.orthogonalize_workspace_bytes(*shape), dtype=torch.uint8, device=DEV)
    vcnn.orthogonalize(*shape, 1, g, out, ws)
    torch.cuda.synchronize()
    del ws
    rows = (lambda m, a, b: m[a:b].t()) if tall else (lambda m, a, b: m[:, a:b])  # columns a .. b of X
    gram = torch.zeros(small, small, dtype=torch.float64, device=DEV)
    step = 1 << 21
    for a in range(0, large, step):
        p = rows(g, a, a + step).double().contiguous()
        gram += torch.mm(p, p.t().contiguous())
    norm2 = torch.diagonal(gram).sum()
    gram /= norm2
    p = A * torch.eye(small, dtype=torch.float64, device=DEV) + B * gram + C * torch.mm(gram, gram)
    for a in (0, large - 1000):
        x = rows(g, a, a + 1000).double() / norm2.sqrt()
        got = rows(out, a, a + 1000).double()
        # columns of X are 1 / sqrt(large) of it each: their share of the bound on all of them
        assert float(torch.linalg.vector_norm(got - torch.mm(p, x.contiguous()))) <= bound(small, large, 1) * (1000 / large) ** 0.5
