"""Orthogonalised updates on the GPU against the oracle in binary64.

A stored pair is within 2^-21 of its number (two roundings of 2^-11 each), or within 2^-39: the low part's subnormal numbers lie 2^-24 apart, of which a
rounding is off by half, and stand for 2^-14 of themselves.  Low low products that are left out another 2^-22.  A sum of k products is one of 3 k / 32 matrix instructions' results, each rounded
(or cut) by 2^-23: summed(k) = (3 k / 32 + 8) 2^-23 + 3 2^-21 of the sum of the magnitudes.  The oracle follows these through the steps."""
import numpy as np
import pytest
import torch

from gpu_util import DEV, say
from oracle import update_oracle as O
from paper_1901_08227_amd import binding as B
from paper_1901_08227_amd import lowbit, update
from test_gpu_lowbit import TYPES, host, normal, same, spread

pytestmark = pytest.mark.gpu

QUINTIC = (update.QUINTIC,) * 5
CUBIC = ((1.5, -0.5, 0.0),) * 3
ONE = (update.QUINTIC,)
SHAPES = [(1, 1, 1), (1, 1, 7), (2, 9, 1), (3, 5, 8), (2, 31, 33), (1, 64, 64), (2, 65, 32), (1, 100, 257), (5, 130, 96), (1, 300, 200), (40, 64, 130), (2, 33, 512), (1, 63, 257), (3, 32, 1024), (2, 20, 600), (2, 64, 513), (1, 32, 1025), (2, 96, 256), (1, 65, 129), (2, 96, 257), (3, 128, 128), (1, 97, 100),
          (1, 128, 129)]


def roundings():
    return 2.0 ** -21, 2.0 ** -39, lambda k: (3 * k / 32 + 8) * 2.0 ** -23 + 3 * 2.0 ** -21


def near(got, x, coefficients, eps, scale):
    got = got.double().cpu().numpy()
    half = torch.finfo(torch.float32).eps / 2
    for g, a in zip(got, x):
        want, error = O.orthogonalize(a, coefficients, eps, scale, roundings())
        if not np.linalg.norm(g - want) <= error + half * np.linalg.norm(want):
            return False
    return True


@pytest.mark.parametrize("coefficients", [QUINTIC, CUBIC, ONE])
@pytest.mark.parametrize("shape", SHAPES)
def test_against_binary64(shape, coefficients):
    x = normal(shape, torch.float32, 1, 1e-3)
    y = update.orthogonalize(x, coefficients, eps=1e-7, scale=1.25)
    assert near(y, host(x), coefficients, 1e-7, 1.25)
    out = spread(torch.zeros_like(x), 0)
    assert update.orthogonalize(spread(x, 0), coefficients, scale=1.25, out=out) is out and torch.equal(out, y)
    assert torch.equal(update.orthogonalize(x, coefficients, scale=1.25), y)
    a = x.clone()
    assert update.orthogonalize(a, coefficients, scale=1.25, out=a) is a and torch.equal(a, y)
    assert torch.equal(update.orthogonalize(x[0], coefficients, scale=1.25), y[0])
    # a turned matrix's result is the result turned (sums of other orders: both are near)
    assert near(update.orthogonalize(x.transpose(1, 2).contiguous(), coefficients, scale=1.25).transpose(1, 2), host(x), coefficients, 1e-7, 1.25)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("to", TYPES)
def test_types(dtype, to):
    x = normal((2, 70, 150), dtype, 2)
    wide = update.orthogonalize(x.float())
    out = torch.empty(x.shape, dtype=to, device=DEV)
    assert same(update.orthogonalize(x, out=out), wide.to(to).cpu())
    assert update.orthogonalize(x).dtype == dtype


def step_in(x, coefficients, eps=1e-7):
    """By the library's products, in x's type."""
    v = x / (x.norm() + eps)
    for a, b, c in coefficients:
        g = v @ v.t()
        v = a * v + (b * g + c * (g @ g)) @ v
    return v


# tiles of all sizes, whole ones and edges, and depths that several workgroups share: few rows and long ones, more tiles than CUs, the largest
@pytest.mark.parametrize("shape", [(1, 70, 5000), (2, 200, 3000), (9, 700, 777), (1, 1100, 1030), (3, 500, 2600), (1, 2100, 1800), (1, 4100, 3900)])
@pytest.mark.parametrize("steps", [1, 5])
def test_large(shape, steps):
    x = normal(shape, torch.float32, 3)
    say(f"update: {shape}, {steps} steps")
    y = update.orthogonalize(x, QUINTIC[:steps])
    z = update.orthogonalize(x.transpose(1, 2).contiguous(), QUINTIC[:steps]).transpose(1, 2)
    for k in {0, shape[0] - 1}:
        want, plain = step_in(x[k].double(), QUINTIC[:steps]), step_in(x[k], QUINTIC[:steps])
        # as accurate as binary32 itself within a factor of four (pairs hold 22 bits where it holds 24); where a step's sums are little more than one product,
        # a X, which binary32 rounds twice, three of the pairs' 2^-22 show: X's, P's, and the low low products that are left out
        for got in (y[k], z[k]):
            assert (got - want).norm() <= 4 * (plain - want).norm() + 3 * 2.0 ** -22 * want.norm()


@pytest.mark.parametrize("size", [1e-30, 1e-9, 1.0, 1e30])
def test_sizes_of_the_input(size):
    x = normal((1, 40, 60), torch.float32, 4).clamp(-3, 3) * size
    assert near(update.orthogonalize(x, QUINTIC, eps=1e-30), host(x), QUINTIC, 1e-30, 1.0)
    assert near(update.orthogonalize(x, QUINTIC, eps=0.5), host(x), QUINTIC, 0.5, 1.0)


def test_one_direction_and_zeros_and_what_is_not_finite():
    x = normal((4, 50, 80), torch.float32, 5)
    x[1] = torch.outer(normal((50,), torch.float32, 6), normal((80,), torch.float32, 7))  # its singular value begins at 1
    x[2] = 0
    clean = update.orthogonalize(x)
    assert near(clean[:2], host(x[:2]), QUINTIC, 1e-7, 1.0) and clean[2].eq(0).all()
    bad = x.clone()
    bad[0, 3, 3], bad[3, 49, 79] = float("inf"), float("nan")
    got = update.orthogonalize(bad)
    assert got[[0, 3]].isnan().all() and torch.equal(got[1:3], clean[1:3])


def test_broadcast_and_nothing_and_refusals():
    x = normal((30, 20), torch.bfloat16, 8)
    got = update.orthogonalize(x.expand(3, 30, 20))
    assert torch.equal(got, update.orthogonalize(x).expand(3, 30, 20))
    for shape in ((0, 5), (5, 0), (2, 0, 5)):
        assert update.orthogonalize(torch.empty(shape, device=DEV)).shape == shape
    with pytest.raises(B.TngError):
        update.orthogonalize(x, ((2.5, 0.0, 0.0),))
    with pytest.raises(ValueError):
        update.orthogonalize(x, ((1.5, 0.0),))
    with pytest.raises(ValueError):
        update.orthogonalize(x, out=torch.empty((30, 21), device=DEV))
    with pytest.raises(TypeError):
        update.orthogonalize(x.to(torch.int8))


def test_graph_and_another_stream():
    x = normal((3, 100, 90), torch.float32, 9)
    want = update.orthogonalize(x)
    side, graph = torch.cuda.Stream(), torch.cuda.CUDAGraph()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        got = update.orthogonalize(x)
    torch.cuda.current_stream().wait_stream(side)
    assert torch.equal(got, want)
    with torch.cuda.graph(graph):
        got = update.orthogonalize(x)
    for k in range(3):
        x.copy_(normal(x.shape, torch.float32, 20 + k))
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(got, update.orthogonalize(x))


def test_ctypes_way_is_the_same(monkeypatch):
    x = normal((2, 70, 90), torch.bfloat16, 40)
    want = update.orthogonalize(x, scale=2)
    monkeypatch.setattr(B, "_layer", B._through_ctypes)
    assert torch.equal(update.orthogonalize(x, scale=2), want)


# few rows of matrices that are too long for one workgroup; alone, a matrix's sums may be taken in other pieces: near as well
@pytest.mark.parametrize("shape", [(2, 1, 2000), (3, 2, 65536), (2, 3, 4097), (70, 33, 1030)])
def test_few_long_rows(shape):
    x = normal(shape, torch.float32, 1, 1e-3)
    y = update.orthogonalize(x, scale=1.25)
    assert near(y, host(x), QUINTIC, 1e-7, 1.25) and torch.equal(update.orthogonalize(x, scale=1.25), y)
    assert near(update.orthogonalize(x[:1], scale=1.25), host(x[:1]), QUINTIC, 1e-7, 1.25)
    assert near(update.orthogonalize(x.transpose(1, 2).contiguous(), scale=1.25).transpose(1, 2), host(x), QUINTIC, 1e-7, 1.25)


# with those above: each product by every kind of tiles that the estimate takes for it, whole ones and such as several workgroups share
@pytest.mark.parametrize("shape", [(1, 2900, 2891), (15, 915, 949), (3, 1162, 1109), (1, 2544, 1603), (15, 873, 595), (2, 1795, 2372)])
def test_all_kinds_of_tiles(shape):
    test_large(shape, 2)


# strips of 128, 256 and 512 columns, the last one whole or not, for 32, 64 and 96 rows; more matrices than strips are for
@pytest.mark.parametrize("shape", [(3, 5, 1100), (2, 20, 3000), (1, 32, 8192), (1, 40, 2500), (2, 64, 8000), (1, 33, 8193), (1, 70, 1000), (2, 96, 2100), (40, 66, 900)])
@pytest.mark.parametrize("steps", [1, 2, 5])
def test_strips(shape, steps):
    coefficients = QUINTIC[:steps]
    for x in (normal(shape, torch.float32, 1, 1e-3), normal(shape, torch.float32, 2, 1e-3).transpose(1, 2).contiguous()):
        y = update.orthogonalize(x, coefficients, scale=1.25)
        wide = x.shape[1] < x.shape[2]
        assert near(y if wide else y.transpose(1, 2), host(x) if wide else host(x.transpose(1, 2).contiguous()), coefficients, 1e-7, 1.25)
        a = x.clone()
        assert update.orthogonalize(a, coefficients, scale=1.25, out=a) is a and torch.equal(a, y)
        out = spread(torch.zeros_like(x), 0)
        assert update.orthogonalize(spread(x, 0), coefficients, scale=1.25, out=out) is out and torch.equal(out, y)
        b = x.bfloat16()
        assert same(update.orthogonalize(b, coefficients), update.orthogonalize(b.float(), coefficients).bfloat16().cpu())


# a strip's launches, those of tiles, and of tiles that several workgroups share
@pytest.mark.parametrize("shape", [(3, 50, 1300), (3, 300, 500), (3, 120, 3000)])
def test_every_way_captured_and_with_what_is_not_finite(shape):
    x = normal(shape, torch.float32, 50)
    bad = x.clone()
    bad[0, 3, 7], bad[1] = float("nan"), 0
    got, want = update.orthogonalize(bad), update.orthogonalize(x)
    assert got[0].isnan().all() and got[1].eq(0).all() and torch.equal(got[2], want[2])
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        first, second = update.orthogonalize(x), update.orthogonalize(bad)
    for k in range(3):
        x.copy_(normal(shape, torch.float32, 60 + k))
        bad.copy_(normal(shape, torch.float32, 70 + k))
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(first, update.orthogonalize(x)) and torch.equal(second, update.orthogonalize(bad))
