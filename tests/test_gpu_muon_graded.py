"""Newton-Schulz products of matrices whose rows or columns are of very different sizes, each row and column against itself.

a X and B X scale row by row and column by column, and float products keep a row of 1e-10 to its own accuracy.  So do the
kernels.  Tolerances: an operand of two f16 terms is off by up to 2^-23 where a float is by 2^-24, and a product leaves out
lo lo, up to 2^-22, where a float's is rounded by 2^-24: the worst row (and column) may be off by four times what the same
products in float arithmetic are, whose sums are rounded as often.  Matrices with one entry a row (the scalar map) are held
to a bound of their own: a step's terms a s, b s^3, c s^5 are off by one, three, five times 2^-22 of themselves, and an
error made before it is multiplied by the map's slope."""
import pytest
import torch

from paper_1501_07338_amd import vcnn
from test_gpu_muon import A, B, C, DEV, matrix, orthogonal, products, workspace


def graded(kind, rows, cols, decades, seed=1):
    gen = torch.Generator().manual_seed(seed)
    g = torch.randn(rows, cols, generator=gen, dtype=torch.float64)
    if kind == "parallel":  # rows of one direction and a little of their own, from 1 down
        g = torch.randn(1, cols, generator=gen, dtype=torch.float64) + 1e-2 * g
    if kind != "columns":
        g *= 10.0 ** (-decades * torch.linspace(0, 1, rows, dtype=torch.float64))[torch.randperm(rows, generator=gen)][:, None]
    if kind in ("columns", "both"):
        g *= 10.0 ** (-decades * torch.linspace(0, 1, cols, dtype=torch.float64))[torch.randperm(cols, generator=gen)][None]
    return g.float()


def worst(got, want):
    """Of a row against itself, and of a column."""
    d = got.double() - want
    return [float((torch.linalg.vector_norm(d, dim=i) / torch.linalg.vector_norm(want, dim=i)).max()) for i in (1, 0)]


@pytest.mark.gpu
@pytest.mark.parametrize("kind", ["rows", "columns", "both", "parallel"])
@pytest.mark.parametrize("decades", [6, 10, 16])
@pytest.mark.parametrize("rows,cols", [(200, 500), (500, 200), (40, 300), (300, 40), (130, 2600), (700, 650), (64, 64), (5, 9000)])
def test_every_row_and_column_keeps_its_accuracy(rows, cols, decades, kind):
    g = graded(kind, rows, cols, decades)
    want = products(g.double(), 5)
    off, plain = worst(orthogonal(g), want), worst(products(g, 5), want)
    assert off[0] <= 4 * max(plain[0], 2.0 ** -22) and off[1] <= 4 * max(plain[1], 2.0 ** -22)


@pytest.mark.gpu
@pytest.mark.parametrize("kind", ["rows", "columns"])
@pytest.mark.parametrize("rows,cols", [(70, 200), (150, 80), (40, 120), (64, 20)])
def test_down_to_the_end_of_the_float_range(rows, cols, kind):
    test_every_row_and_column_keeps_its_accuracy(rows, cols, 33, kind)


@pytest.mark.gpu
@pytest.mark.parametrize("rows,cols", [(1400, 1500), (2200, 1300), (1100, 4100)])
def test_larger_tiles(rows, cols):
    """Sizes of the 128-wide tiles and of the shared sums."""
    g = graded("both", rows, cols, 10).to(DEV)
    want = products(g.double(), 5)
    out = torch.empty_like(g)
    vcnn.orthogonalize(rows, cols, 5, g, out, workspace(vcnn.orthogonalize_workspace_bytes(rows, cols)))
    off, plain = worst(out, want), worst(products(g, 5), want)
    assert off[0] <= 4 * plain[0] and off[1] <= 4 * plain[1]


@pytest.mark.gpu
@pytest.mark.parametrize("steps", [1, 5, 8, 24, 32])
@pytest.mark.parametrize("rows,cols", [(80, 120), (150, 90), (50, 90), (64, 64)])
def test_the_scalar_map_of_small_entries(rows, cols, steps):
    n = min(rows, cols)
    s = 10.0 ** -torch.linspace(0, 12, n, dtype=torch.float64)
    i, j = torch.arange(n) + (rows - n), torch.arange(n) + (cols - n)
    g = torch.zeros(rows, cols)
    g[i, j] = s.float()
    got = orthogonal(g, steps)
    v = g[i, j].double()
    v /= torch.linalg.vector_norm(v)
    off = v * 2.0 ** -23
    for _ in range(steps):
        slope = (A + 3 * B * v ** 2 + 5 * C * v ** 4).abs()
        off = off * slope + 2.0 ** -22 * (A * v + 3 * -B * v ** 3 + 5 * C * v ** 5)
        v = A * v + B * v ** 3 + C * v ** 5
    assert bool(((got[i, j].double() - v).abs() <= off).all())
    assert int((got != 0).sum()) == n


@pytest.mark.gpu
@pytest.mark.parametrize("shapes", [[(60, 300), (300, 500), (20, 20)], [(60, 300), (10, 64), (20, 20)]], ids=["with a large one", "small"])
def test_update_beside_others(shapes):
    gs = [graded("rows", *s, 10, seed=i) for i, s in enumerate(shapes)]
    ws, ms = ([torch.zeros(s, device=DEV) for s in shapes] for _ in range(2))
    vcnn.muon_update_multi(-1.0, 0.0, False, 0.0, 5, ws, [g.to(DEV) for g in gs], ms, workspace(vcnn.muon_workspace_bytes(shapes)))
    for g, w in zip(gs, ws):
        want = products(g.double(), 5) * max(1.0, g.shape[0] / g.shape[1]) ** 0.5
        off, plain = worst(w.cpu(), want), worst(products(g, 5), products(g.double(), 5))
        assert off[0] <= 4 * max(plain[0], 2.0 ** -22) and off[1] <= 4 * max(plain[1], 2.0 ** -22)


@pytest.mark.gpu
def test_rows_and_columns_of_zeros():
    g = matrix(8, 150, 260)
    g[[0, 77, 149]] = 0.0
    g[:, [3, 128, 259]] = 0.0
    out = orthogonal(g)
    assert bool((out[[0, 77, 149]] == 0).all()) and bool((out[:, [3, 128, 259]] == 0).all())
    want = products(g.double(), 5)
    off, plain = torch.linalg.vector_norm(out.double() - want), torch.linalg.vector_norm(products(g, 5).double() - want)
    assert float(off) <= 2 * float(plain)
