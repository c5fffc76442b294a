"""The norm where its sums are delicate: squares below the float range.  Tolerances are those of test_gpu_norm."""
import pytest
import torch

from paper_1501_07338_amd import vcnn
from test_gpu_norm import U, Guarded, depth, dev, gain_of, tensor


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
