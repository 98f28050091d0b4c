"""Root-mean-square norms on the GPU against the oracle in binary64.

Tolerances, in units u = 2^-24 of binary32.  A row's sum of squares is made by lanes that add at most 48 squares one after another (rows of up to
40000 columns in these tests), six steps over a wavefront and sixteen over a workgroup: at most 72 roundings with the squares' own, all of one sign,
so 72 u of the sum; halved by the root, and with the mean, the root and the quotient: s is within 40 u.  y = (h s) w: two more.
A dot product is within 75 u of the sum of its magnitudes.  To that comes half a step of the result's type."""
import numpy as np
import pytest
import torch

from gpu_util import DEV
from oracle import token_oracle as O
from paper_1901_08227_amd import binding as B
from paper_1901_08227_amd import lowbit
from test_gpu_lowbit import TINIEST, TYPES, host, normal, same, spread

pytestmark = pytest.mark.gpu

U = 2.0 ** -24
HALF_STEP = {t: torch.finfo(t).eps / 2 for t in TYPES}
S = 40 * U  # of s
SHAPES = [(1, 1, 1), (2, 3, 5), (1, 1, 8), (3, 2, 13), (2, 33, 64), (2, 17, 250), (1, 5, 513), (2, 600, 1000), (1, 1100, 2047), (1, 4, 2048), (1, 3, 4096), (2, 2, 8191),
          (1, 2, 16000), (1, 3, 20011), (1, 2, 32768), (2, 2, 40003)]
EPS = 1e-5


def weights(cols, seed=9):
    return 1 + 0.3 * normal((cols,), torch.float32, seed)


def added(x, r):
    """h as it is stored."""
    return (x.float() + r.float()).to(x.dtype)


def near(got, want, error, dtype):
    """|got - want| within error and half a step of the type."""
    got, off = got.double().cpu().numpy(), None
    off = np.abs(got - want)
    return bool(np.all(off <= error + HALF_STEP[dtype] * (np.abs(want) + error) + TINIEST[dtype]))


def y_near(got, h, w, eps, dtype):
    want = O.rms_norm(host(h), None if w is None else host(w), eps)
    return near(got, want, (S + 2 * U) * np.abs(want), dtype)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("shape", SHAPES)
def test_norm(shape, dtype):
    x, r, w = normal(shape, dtype, 1, 3.0), normal(shape, dtype, 2), weights(shape[2])
    for a, b in ((x, r), (spread(x, 0), spread(r, 0)), (x, spread(r, 0))):
        assert y_near(lowbit.rms_norm(a, w, eps=EPS), x, w, EPS, dtype)
        y, h = lowbit.rms_norm(a, w, residual=b, eps=EPS)
        assert same(h, added(x, r).cpu()) and y_near(y, h, w, EPS, dtype)
        # the same, bit for bit, as the norm of the sum; without weights as with ones
        assert same(lowbit.rms_norm(h, w, eps=EPS), y.cpu())
        assert same(lowbit.rms_norm(a, eps=EPS), lowbit.rms_norm(x, torch.ones_like(w), eps=EPS).cpu())
        out = spread(torch.zeros_like(x), 0)
        assert lowbit.rms_norm(a, w, residual=b, eps=EPS, out=out)[0] is out and same(out, y.cpu())


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("shape", SHAPES)
def test_codes(shape, dtype):
    x, r, w = normal(shape, dtype, 3, 2.0), normal(shape, dtype, 4), weights(shape[2])
    n = lowbit.rms_norm_codes(spread(x, 0), w, residual=r, eps=EPS, turned=True)
    assert same(n.h, added(x, r).cpu()) and n.q.shape == shape and n.scale.shape == shape[:2]
    assert torch.equal(n.qt, n.q.transpose(1, 2))
    want = O.rms_norm(host(n.h), host(w), EPS)
    step = np.abs(want).max(-1, keepdims=True) / 127
    # the scale: y's error, and the quotient's; a place on the scale of codes: 127 times y's error, the scale's inverse's and three roundings
    assert np.all(np.abs(n.scale.double().cpu().numpy()[..., None] - step) <= (S + 4 * U) * step)
    assert np.all(np.abs(n.q.double().cpu().numpy() - want / step) <= 0.5 + 127 * (2 * S + 8 * U))
    if dtype == torch.float32:  # (y is rounded nowhere on the way)
        q, scale, qt = lowbit.quantize_rows(lowbit.rms_norm(n.h, w, eps=EPS), turned=True)
        assert torch.equal(q, n.q) and torch.equal(scale, n.scale) and torch.equal(qt, n.qt)
    again = lowbit.rms_norm_codes(n.h, w, eps=EPS)
    assert again.h is n.h and again.qt is None and torch.equal(again.q, n.q) and torch.equal(again.scale, n.scale)


def grad_near(dx, dw, dy, h, w, eps, r, dtype):
    a = [host(t) if t is not None else None for t in (dy, h, w, r)]
    want, want_dw = O.rms_norm_grad(a[0], a[1], a[2], eps, a[3])
    s = 1 / np.sqrt(O.mean_square(a[1].astype(np.float64)) + eps)
    unit, g = np.abs(a[1] * s), np.abs(a[0] * (1.0 if a[2] is None else a[2].astype(np.float64)))
    along = np.mean(g * unit, -1, keepdims=True)
    # s g, the part along h (dot product, s twice, three products) and the sum with the residual's
    error = (S + 4 * U) * s * g + (75 * U + 3 * S + 6 * U) * s * unit * along + 2 * U * np.abs(want) + (0 if r is None else 2 * U * np.abs(a[3]))
    assert near(dx, want, error, dtype)
    if dw is not None:
        size = np.sum(np.abs(a[0]) * unit, -2)
        rows = dy.shape[-2]
        assert np.all(np.abs(dw.double().cpu().numpy() - want_dw) <= (S + (4 + rows) * U) * size + 2.0 ** -149 * rows)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("shape", SHAPES)
def test_gradient(shape, dtype):
    h, dy, r, w = normal(shape, dtype, 5, 2.0), normal(shape, dtype, 6), normal(shape, dtype, 7), weights(shape[2])
    dx, dw = lowbit.rms_norm_grad(dy, h, w, dresidual=r, eps=EPS)
    assert dw.shape == (shape[0], shape[2])
    grad_near(dx, dw, dy, h, w, EPS, r, dtype)
    sdx, sdw = lowbit.rms_norm_grad(spread(dy, 0), spread(h, 0), w, dresidual=spread(r, 0), eps=EPS, out=spread(torch.zeros_like(h), 0))
    assert same(sdx, dx.cpu()) and torch.equal(sdw, dw)
    plain, none = lowbit.rms_norm_grad(dy, h, eps=EPS)
    assert none is None
    grad_near(plain, None, dy, h, None, EPS, None, dtype)
    # results where inputs are
    for k in range(3):
        a = [t.clone() for t in (dy, h, r)]
        got, got_dw = lowbit.rms_norm_grad(a[0], a[1], w, dresidual=a[2], eps=EPS, out=a[k])
        assert got is a[k] and same(got, dx.cpu()) and torch.equal(got_dw, dw)


@pytest.mark.parametrize("cols", [5, 100, 1500, 5000, 10000, 20011, 40003])
def test_in_place(cols):
    x, r, w = normal((2, 9, cols), torch.bfloat16, 10), normal((2, 9, cols), torch.bfloat16, 11), weights(cols)
    y, h = lowbit.rms_norm(x, w, residual=r)
    for at in (0, 1):  # y where an input is
        a = [x.clone(), r.clone()]
        got, got_h = lowbit.rms_norm(a[0], w, residual=a[1], out=a[at])
        assert same(got, y.cpu()) and same(got_h, h.cpu())
    a = x.clone()
    assert same(lowbit.rms_norm(a, w, out=a), lowbit.rms_norm(x, w).cpu())
    M, R, C = x.shape  # h where an input is
    for at in (0, 1):
        a = [x.clone(), r.clone(), torch.empty_like(x)]
        mats = [lowbit._matrix(t, lowbit._TYPES, "x") for t in a]
        B._check(B.lib().tng_rms_norm(lowbit._stream(x.device), mats[0], mats[1], B.TngRms(w.data_ptr(), 1e-6), mats[at], mats[2]), "tng_rms_norm")
        assert same(a[at], h.cpu()) and same(a[2], y.cpu())


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("cols", [40, 1500, 20011, 40003])
def test_values_far_from_one(dtype, cols):
    big = {torch.float32: 2.0 ** 100, torch.bfloat16: 2.0 ** 100, torch.float16: 2.0 ** 10}[dtype]
    h, dy, w = normal((1, 4, cols), dtype, 12), normal((1, 4, cols), dtype, 13), weights(cols)
    h[0, 0] *= big
    h[0, 1] = 0
    h[0, 2] *= 2.0 ** -12  # (mean squares about eps and below)
    assert y_near(lowbit.rms_norm(h, w, eps=1e-8), h, w, 1e-8, dtype)
    n = lowbit.rms_norm_codes(h, w, eps=1e-8)
    assert n.scale.isfinite().all() and n.scale[0, 1] == 0 and not n.q[0, 1].any()
    dx, dw = lowbit.rms_norm_grad(dy, h, w, eps=1e-8)
    # (a row of large numbers has gradients that its type may not hold: 2^-100 of bfloat16 and float32 is held, so they are compared too)
    grad_near(dx, dw, dy, h, w, 1e-8, None, dtype)


@pytest.mark.parametrize("cols", [7, 300, 5000, 20011, 40003])
def test_a_row_that_is_not_finite_is_nan_and_no_other(cols):
    x, dy, w = normal((1, 5, cols), torch.bfloat16, 14), normal((1, 5, cols), torch.bfloat16, 15), weights(cols)
    bad = x.clone()
    bad[0, 1, cols // 2] = float("inf")
    bad[0, 3, cols - 1] = float("nan")
    for got, want in ((lowbit.rms_norm(bad, w), lowbit.rms_norm(x, w)), (lowbit.rms_norm_grad(dy, bad, w)[0], lowbit.rms_norm_grad(dy, x, w)[0])):
        assert got[0, [1, 3]].isnan().all() and torch.equal(got[0, [0, 2, 4]], want[0, [0, 2, 4]])
    scale = lowbit.rms_norm_codes(bad, w).scale
    assert scale[0, [1, 3]].isnan().all() and scale[0, [0, 2, 4]].isfinite().all()


def test_one_worker_broadcast_inputs_and_nothing():
    x, w = normal((6, 70), torch.float16, 16), weights(70)
    assert same(lowbit.rms_norm(x, w), lowbit.rms_norm(x[None], w)[0].cpu())
    dx, dw = lowbit.rms_norm_grad(x, x, w)
    assert dw.shape == (70,)
    row = normal((1, 1, 70), torch.float16, 17)
    wide = row.expand(3, 6, 70)
    assert same(lowbit.rms_norm(wide, w, residual=x.expand(3, 6, 70))[0], lowbit.rms_norm(wide.contiguous(), w, residual=x.expand(3, 6, 70).contiguous())[0].cpu())
    got, want = lowbit.rms_norm_grad(wide, x.expand(3, 6, 70), w), lowbit.rms_norm_grad(wide.contiguous(), x.expand(3, 6, 70).contiguous(), w)
    assert same(got[0], want[0].cpu()) and torch.equal(got[1], want[1])
    none = torch.empty((2, 0, 70), device=DEV)
    y, h = lowbit.rms_norm(none, w, residual=none)
    assert y.shape == h.shape == none.shape and lowbit.rms_norm_codes(none, w, turned=True).qt.shape == (2, 70, 0)
    assert lowbit.rms_norm_grad(none, none, w)[1].eq(0).all()
    empty = torch.empty((2, 5, 0), device=DEV)
    assert lowbit.rms_norm(empty).shape == empty.shape and lowbit.rms_norm_codes(empty).scale.eq(0).all()
    with pytest.raises(B.TngError):
        lowbit.rms_norm(x, w, eps=0.0)
    with pytest.raises(ValueError):
        lowbit.rms_norm(x, w[:69])
    with pytest.raises(B.TngError):
        lowbit.rms_norm(x, w, residual=x[:5])


def test_rows_that_alternate_between_workers_are_refused():
    x = normal((6, 2, 40), torch.float32, 18).transpose(0, 1)
    with pytest.raises(B.TngError):
        lowbit.rms_norm(x)


def test_graph_and_another_stream():
    x, r, w, dy = (normal((2, 300, 1000), torch.bfloat16, k) for k in (20, 21, 22, 23))
    w = weights(1000)
    n = lowbit.rms_norm_codes(x, w, residual=r, turned=True)
    dx, dw = lowbit.rms_norm_grad(dy, n.h, w, dresidual=r)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.stream(side):
        got = lowbit.rms_norm_grad(dy, n.h, w, dresidual=r)
    torch.cuda.current_stream().wait_stream(side)
    assert torch.equal(got[0], dx) and torch.equal(got[1], dw)
    with torch.cuda.graph(graph):
        gn = lowbit.rms_norm_codes(x, w, residual=r, turned=True)
        gdx, gdw = lowbit.rms_norm_grad(dy, gn.h, w, dresidual=r)
    for k in range(3):
        x.copy_(normal(x.shape, torch.bfloat16, 30 + k))
        graph.replay()
        torch.cuda.synchronize()
        n = lowbit.rms_norm_codes(x, w, residual=r, turned=True)
        dx, dw = lowbit.rms_norm_grad(dy, n.h, w, dresidual=r)
        assert all(torch.equal(a, b) for a, b in zip((*gn, gdx, gdw), (*n, dx, dw)))


def test_ctypes_way_is_the_same(monkeypatch):
    x, r, w = normal((2, 30, 100), torch.bfloat16, 40), normal((2, 30, 100), torch.bfloat16, 41), weights(100)
    calls = lambda: (*lowbit.rms_norm(x, w, residual=r), lowbit.rms_norm(x), *lowbit.rms_norm_codes(x, w, residual=r, turned=True),  # noqa: E731
                     *lowbit.rms_norm_grad(x, r, w, dresidual=r))
    want = calls()
    monkeypatch.setattr(B, "_layer", B._through_ctypes)
    assert all(torch.equal(a, b) for a, b in zip(calls(), want))


@pytest.mark.parametrize("rows,cols", [((1 << 19) + 1, 8200), (3, 40000)])
def test_more_rows_than_a_side_of_a_grid(rows, cols):
    # eight workers of more than 2^19 rows: beyond 2^32 threads; one row stands for all
    x, w = normal((1, 1, cols), torch.bfloat16, 60), weights(cols)
    n, one = lowbit.rms_norm_codes(x.expand(8, rows, cols), w), lowbit.rms_norm_codes(x, w)
    assert n.scale.eq(one.scale).all()
    for m in range(8):
        assert n.q[m].eq(one.q[0]).all()
