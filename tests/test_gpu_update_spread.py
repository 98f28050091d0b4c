"""Orthogonalised updates of matrices whose rows, columns or elements are of very different sizes: every row and every column of the result, by itself, as near
to binary64's as binary32's are.

The measure is the worst row's (column's) error over that row's norm: four times what the same steps in binary32 have there, and 3 2^-22 for the roundings of
operands to 22 bits, as in test_gpu_update_binary32.py.  Binary32's sums are made as often as the kernels': a sum of k products is k / 32 times three matrix
instructions' results, one after another, each of which rounds.  That counts where a row's sum is of one sign and what it is taken from leaves little: of one large
column a + b + c = 0.70 of 3.44 is left, five times the sum's error; k = 1030 are 99 roundings, of half a last place 2^-24 each at random
sqrt(99 / 3) 2^-24 = 3.4e-7 in each of two products (G G, E X), against a library's order of unknown length that has a third of it."""
import math

import pytest
import torch

from gpu_util import DEV, say
from paper_1901_08227_amd import update
from test_gpu_lowbit import normal
from test_gpu_update import CUBIC, QUINTIC, step_in

pytestmark = pytest.mark.gpu

# one launch of every kind, strips of every kind, tiles of 64, 128, 192 and 256, and such as several workgroups share
SHAPES = [(1, 20, 30), (2, 32, 900), (1, 50, 70), (1, 64, 400), (2, 64, 256), (1, 90, 200), (1, 120, 128), (2, 30, 1500), (1, 64, 1024), (1, 60, 6000),
          (1, 96, 2100), (2, 130, 200), (1, 120, 3000), (4, 400, 500), (1, 1100, 1030)]
LARGE = [(3, 1162, 1109), (1, 2544, 1603), (1, 2900, 2891)]
KINDS = ["rows 1e-3", "columns 1e-3", "rows 1e-4", "rows 1e-6", "rows 1e-12", "columns 1e-6", "columns 1e-12", "both 1e-6", "one row", "one column", "one element", "steps of rows"]


def falling(n, by):
    """1 to 10^-by, in no order."""
    at = torch.randperm(n, generator=torch.Generator().manual_seed(n)).to(DEV)
    return torch.exp(-by * math.log(10.0) * at / max(1, n - 1)).float()


def spread(shape, kind, seed=1):
    x = normal(shape, torch.float32, seed)
    _, n, m = shape
    what, _, by = kind.rpartition(" ")
    if what == "rows":
        x *= falling(n, -math.log10(float(by)))[:, None]
    elif what == "columns":
        x *= falling(m, -math.log10(float(by)))
    elif what == "both":
        x *= falling(n, -math.log10(float(by)))[:, None] * falling(m, -math.log10(float(by)))
    elif kind == "one row":
        x[:, n // 2] *= 1e5
    elif kind == "one column":
        x[:, :, m // 2] *= 1e5
    elif kind == "one element":
        x[:, n // 2, m // 3] = 1e6
    else:  # (halves: 1 and 1e-9)
        x[:, n // 2:] *= 1e-9
    return x


def product(a, b):
    """a b^T of binary32, summed 32 products at a time, three roundings for each 32."""
    total = torch.zeros(a.shape[0], b.shape[0], device=a.device)
    for k in range(0, a.shape[1], 32):
        third = a[:, k:k + 32].double() @ b[:, k:k + 32].double().t().contiguous() / 3
        for _ in range(3):
            total = (total.double() + third).float()
    return total


def step_in_order(x, coefficients, eps=1e-7):
    v = (x.double() / (x.double().norm() + eps)).float()
    for a, b, c in coefficients:
        g = product(v, v)
        v = a * v + product(b * g + c * product(g, g), v.t())
    return v


def worst(got, want, dim):
    size = want.norm(dim=dim)
    assert (size > 0).all()
    return ((got.double() - want).norm(dim=dim) / size).max().item()


def by_rows_and_columns(got, x, coefficients):
    """One matrix."""
    if x.shape[0] > x.shape[1]:
        got, x = got.t(), x.t().contiguous()
    want, plain = step_in(x.double(), coefficients), step_in_order(x, coefficients)
    for dim in (0, 1):
        off, of_plain = worst(got, want, dim), worst(plain, want, dim)
        assert off <= 4 * of_plain + 3 * 2.0 ** -22, (("columns", "rows")[dim], off, of_plain)


@pytest.mark.parametrize("coefficients", [QUINTIC[:1], QUINTIC[:2], QUINTIC, CUBIC])
@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("shape", SHAPES)
def test_every_row_and_column(shape, kind, coefficients):
    say(f"update: {shape}, {kind}, {len(coefficients)} steps")
    x = spread(shape, kind)
    y = update.orthogonalize(x, coefficients)
    z = update.orthogonalize(x.transpose(1, 2).contiguous(), coefficients).transpose(1, 2)
    for k in {0, shape[0] - 1}:
        by_rows_and_columns(y[k], x[k], coefficients)
        by_rows_and_columns(z[k], x[k], coefficients)


@pytest.mark.parametrize("kind", ["rows 1e-6", "columns 1e-6"])
@pytest.mark.parametrize("shape", LARGE)
def test_every_row_and_column_of_large_ones(shape, kind):
    by_rows_and_columns(update.orthogonalize(spread(shape, kind), QUINTIC[:2])[0], spread(shape, kind)[0], QUINTIC[:2])


# norms that shrink first, that grow for long, that nothing happens to; each step's products by whole numbers that binary32 holds as well as binary64
@pytest.mark.parametrize("coefficients", [((0.5, 0.0, 0.0),) * 8 + QUINTIC, ((1.5, -0.5, 0.0),) * 10, ((1.0, 0.0, 0.0),) * 64, ((0.0, 1.0, 0.0),) * 2, ((0.0, 0.0, 1.0),)])
@pytest.mark.parametrize("shape", [(1, 20, 30), (1, 64, 1024), (1, 130, 200)])
def test_other_schedules(shape, coefficients):
    for kind in ("even", "rows 1e-4"):
        x = spread(shape, kind) if kind != "even" else normal(shape, torch.float32, 1)
        y = update.orthogonalize(x, coefficients)[0]
        if coefficients[0] == (1.0, 0.0, 0.0):
            assert torch.equal(y, (x[0].double() * (1 / (x[0].double().norm() + float(torch.tensor(1e-7, dtype=torch.float32))))).float())
        else:
            by_rows_and_columns(y, x[0], coefficients)


@pytest.mark.parametrize("shape", [(1, 20, 30), (1, 64, 1024), (1, 130, 200)])
def test_an_eps_beyond_the_matrix(shape):
    """x / (||x|| + eps) of 1e-9 and less: as of any other matrix."""
    x = normal(shape, torch.float32, 3) * 1e-9
    want = x.double() / (x.double().norm() + 1.0)
    for a, b, c in QUINTIC:
        g = want[0] @ want[0].t()
        want = (a * want[0] + (b * g + c * (g @ g)) @ want[0])[None]
    got = update.orthogonalize(x, QUINTIC, eps=1.0)
    assert (got.double() - want).norm() <= 16 * 2.0 ** -24 * want.norm()  # (a X alone: a product and a rounding a step, and the first)


@pytest.mark.parametrize("shape", [(2, 20, 30), (2, 40, 1500), (2, 130, 200)])
def test_rows_and_columns_of_zeros(shape):
    x = normal(shape, torch.float32, 4)
    x[0, 3] = 0
    x[0, :, 5] = 0
    x[1, 1:] = 0
    y = update.orthogonalize(x)
    assert y.isfinite().all() and not y[0, 3].any() and not y[0, :, 5].any() and not y[1, 1:].any()
    keep = [k for k in range(shape[1]) if k != 3], [k for k in range(shape[2]) if k != 5]
    part = x[0][keep[0]][:, keep[1]]
    want, plain = step_in(part.double(), QUINTIC), step_in(part, QUINTIC)
    assert (y[0][keep[0]][:, keep[1]].double() - want).norm() <= 4 * (plain.double() - want).norm() + 3 * 2.0 ** -22 * want.norm()
