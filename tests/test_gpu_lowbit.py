"""The layer calls on the GPU against the oracle: codes, scales, kept elements and dropout bit for bit, products within the
roundings that they are allowed."""
import numpy as np
import pytest
import torch

from gpu_util import DEV, say
from oracle import lowbit_oracle as L
from paper_1901_08227_amd import binding as B
from paper_1901_08227_amd import lowbit

pytestmark = pytest.mark.gpu

TYPES = [torch.float32, torch.bfloat16, torch.float16]
UNIT = {torch.float32: 2.0 ** -24, torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11}
TINIEST = {torch.float32: 2.0 ** -150, torch.bfloat16: 2.0 ** -134, torch.float16: 2.0 ** -25}  # half the smallest subnormal number


def gen(seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    return g


def normal(shape, dtype, seed, scale=1.0):
    return (torch.randn(shape, generator=gen(seed), device=DEV) * scale).to(dtype)


def host(t):
    return t.float().cpu().numpy()


def three(a):
    return a[None] if a.ndim == 2 else a


def spread(t, seed):
    """The same matrix inside a larger one: rows and workers with gaps between them, not 16-byte aligned."""
    M, R, C = t.shape
    big = torch.zeros((M, R + 2, C + 5), dtype=t.dtype, device=t.device)
    view = big[:, 1:R + 1, 3:C + 3]
    view.copy_(t)
    return view


def rounded(x, dtype):
    """float32 numpy -> the type, to nearest even (torch on the host)."""
    return torch.from_numpy(np.ascontiguousarray(x)).to(dtype)


def same(got, want):
    got = got.cpu()
    assert got.shape == want.shape and got.dtype == want.dtype
    return torch.equal(torch.nan_to_num(got, nan=77.0), torch.nan_to_num(want, nan=77.0)) and torch.equal(got.isnan(), want.isnan())


def codes_of(v, n):
    return three(v.cpu().numpy())[..., :n]


# ---- dropout

SHAPES = [(1, 1, 1), (1, 1, 7), (2, 3, 5), (1, 2, 8), (3, 1, 1027), (2, 33, 64), (2, 17, 250), (1, 5, 4099)]


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("shape", SHAPES)
def test_dropout(shape, dtype):
    x, res, dy = normal(shape, dtype, 1, 3.0), normal(shape, dtype, 2), normal(shape, dtype, 3)
    for p, relu in ((0.0, True), (0.1, False), (0.5, True), (0.999, False)):
        d = lowbit.Drop(seed=(5 << 32) + 9, iter=3, site=6, p=p, relu=relu)
        keep = L.kept(d.seed, d.iter, d.site, p, shape)
        for a, r, g in ((x, res, dy), (spread(x, 0), spread(res, 0), spread(dy, 0)), (spread(x, 0), res, dy)):
            assert same(lowbit.dropout(a, d), rounded(L.dropout(host(x), keep, p, relu), dtype)), (p, relu)
            assert same(lowbit.dropout(a, d, r), rounded(L.dropout(host(x), keep, p, relu, host(res)), dtype)), (p, relu)
            want = rounded(L.dropout_grad(host(dy), keep, p, relu, host(x)), dtype)
            assert same(lowbit.dropout_grad(g, d, a), want), (p, relu)
            out = spread(torch.zeros_like(x), 0)
            assert lowbit.dropout_grad(g, d, a, out=out) is out and same(out, want)
            if not relu:
                assert same(lowbit.dropout_grad(g, d), want)


def test_dropout_of_more_than_the_caches_hold():
    shape = (2, 2100, 4099)
    say("layer calls: dropout of 2 x 2100 x 4099")
    x, res = normal(shape, torch.bfloat16, 8), normal(shape, torch.bfloat16, 9)
    d = lowbit.Drop(3, 1, 4, 0.3, True)
    keep = L.kept(3, 1, 4, 0.3, shape)
    assert same(lowbit.dropout(x, d, res), rounded(L.dropout(host(x), keep, 0.3, True, host(res)), torch.bfloat16))
    assert same(lowbit.dropout(x, d), rounded(L.dropout(host(x), keep, 0.3, True), torch.bfloat16))
    assert same(lowbit.dropout_grad(res, d, x), rounded(L.dropout_grad(host(res), keep, 0.3, True, host(x)), torch.bfloat16))


def test_dropout_of_one_worker_in_place_and_broadcast():
    x = normal((40, 66), torch.bfloat16, 4)
    d = lowbit.Drop(1, 2, 3, 0.3)
    want = lowbit.dropout(x[None], d)[0]
    assert same(lowbit.dropout(x, d), want.cpu())
    y = x.clone()
    assert lowbit.dropout(y, d, out=y) is y and same(y, want.cpu())
    # one row, one worker that stand for all: the draws are still those of each element
    row = normal((1, 1, 66), torch.bfloat16, 5)
    assert same(lowbit.dropout(row.expand(3, 40, 66), d), lowbit.dropout(row.expand(3, 40, 66).contiguous(), d).cpu())


@pytest.mark.parametrize("dtype", TYPES)
def test_dropout_of_what_is_not_finite(dtype):
    x = normal((2, 6, 40), dtype, 6)
    x[0, 0, :8] = float("inf")
    x[1, 1, :8] = float("-inf")
    x[0, 2, :8] = float("nan")
    res = normal((2, 6, 40), dtype, 7)
    for relu in (False, True):
        d = lowbit.Drop(1, 2, 3, 0.5, relu)
        keep = L.kept(1, 2, 3, 0.5, (2, 6, 40))
        got = lowbit.dropout(x, d)
        assert same(got, rounded(L.dropout(host(x), keep, 0.5, relu), dtype))
        assert not got.cpu()[torch.from_numpy(~keep)].isnan().any()  # a dropped element is 0 whatever it was
        assert same(lowbit.dropout(x, d, res), rounded(L.dropout(host(x), keep, 0.5, relu, host(res)), dtype))
        assert same(lowbit.dropout_grad(x, d, res), rounded(L.dropout_grad(host(x), keep, 0.5, relu, host(res)), dtype))
        assert same(lowbit.dropout_grad(res, d, x), rounded(L.dropout_grad(host(res), keep, 0.5, relu, host(x)), dtype))


def test_empty_matrices():
    d = lowbit.Drop(1, 2, 3, 0.5)
    for shape in ((2, 0, 8), (2, 8, 0), (0, 8)):
        x = torch.empty(shape, device=DEV)
        assert lowbit.dropout(x, d).shape == shape and lowbit.dropout_grad(x, d).shape == shape
    q, s, qt = lowbit.quantize_rows(torch.empty((2, 3, 0), device=DEV), turned=True)
    assert not s.any() and q.shape == (2, 3, 0) and qt.shape == (2, 0, 3)
    q, s, qt = lowbit.quantize_rows(torch.empty((2, 0, 3), device=DEV), turned=True)
    assert s.shape == (2, 0) and qt.shape == (2, 3, 0)
    got = lowbit.quantize_grad(torch.empty((2, 0, 5), device=DEV), seed=0, iter=0, site=0)
    assert not got[3].any() and not got[4].any() and got[2].shape == (2, 5, 0)
    got = lowbit.quantize_grad(torch.empty((2, 5, 0), device=DEV), seed=0, iter=0, site=0)
    assert not got[1].any() and got[0].shape == (2, 5, 0)
    i8 = dict(dtype=torch.int8, device=DEV)
    bias = torch.arange(5.0, device=DEV)
    y = lowbit.matmul_i8(torch.empty((3, 0), **i8), torch.empty((5, 0), **i8), bias=bias)
    assert torch.equal(y, bias.expand(3, 5))
    assert not lowbit.matmul_i8(torch.empty((2, 3, 0), **i8), torch.empty((2, 5, 0), **i8)).any()
    assert lowbit.matmul_i8(torch.empty((0, 4), **i8), torch.empty((5, 4), **i8)).shape == (0, 5)


# ---- codes

ROWS = [(1, 1, 1), (1, 1, 4096), (2, 3, 5), (1, 127, 17), (1, 129, 16), (2, 64, 130), (1, 300, 257), (3, 2, 2049), (1, 3, 4100),
        (1, 2, 8192), (2, 2, 8205), (1, 130, 1000), (1, 1, 20000)]


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("shape", ROWS)
def test_codes_of_rows(shape, dtype):
    x = normal(shape, dtype, 11)
    for drop in (None, lowbit.Drop(3, 4, 5, 0.25, True), lowbit.Drop(3, 4, 5, 0.0, True), lowbit.Drop(3, 4, 5, 0.5, False)):
        v = host(x)
        if drop is not None:
            v = L.dropped(v, L.kept(3, 4, 5, drop.p, shape), drop.p, drop.relu)
        want, scale = L.codes(v, 2)
        for a in (x, spread(x, 0)):
            q, s, qt = lowbit.quantize_rows(a, drop, turned=True)
            assert np.array_equal(q.cpu().numpy(), want) and np.array_equal(s.cpu().numpy(), scale[..., 0])
            assert np.array_equal(qt.cpu().numpy(), np.swapaxes(want, 1, 2))
            q2, s2 = lowbit.quantize_rows(a, drop)
            assert torch.equal(q2, q) and torch.equal(s2, s)


@pytest.mark.parametrize("cols", [40, 9000])
def test_codes_of_rows_at_the_ends_of_the_range(cols):
    x = torch.zeros((7, cols), device=DEV)
    x[1, 3] = 1e-40                         # subnormal: taken as 0
    x[2, :9] = torch.tensor([1.1754944e-38 * (k + 1) for k in range(9)])
    x[3, 4], x[3, 5] = 3.4e38, -1.7e38
    x[4, 0] = float("inf")
    x[5, -1] = float("nan")
    x[6] = -0.0
    q, s = lowbit.quantize_rows(x)
    want, scale = L.codes(host(x)[None], 2)
    fine = [0, 1, 2, 3, 6]
    assert np.array_equal(q.cpu().numpy()[fine], want[0][fine])
    assert np.array_equal(s.cpu().numpy(), scale[0, :, 0], equal_nan=True) and s[4:6].isnan().all()
    y = lowbit.matmul_i8(q, q, s)
    assert y[4:6].isnan().all() and not y[fine].isnan().any()


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("shape", [(1, 1, 1), (1, 1, 512), (2, 3, 5), (1, 129, 516), (2, 128, 128), (3, 300, 257), (1, 513, 1026), (2, 7, 1030)])
def test_codes_of_a_gradient(shape, dtype):
    M, T, N = shape
    dy = normal(shape, dtype, 21, 1e-2)
    if T > 2:
        dy[0, 1] = 0.0                       # a row, and a column, that hold nothing
        dy[0, :, N // 2] = 0.0
    cs = torch.rand(N, generator=gen(22), device=DEV) + 0.5
    rs = torch.rand((M, T), generator=gen(23), device=DEV) + 0.5
    for a, c, r in ((dy, cs, rs), (spread(dy, 0), cs, rs), (dy, None, None)):
        got = lowbit.quantize_grad(a, c, r, seed=77, iter=8, site=9)
        q, qs, qt, qts = L.grad_codes(host(dy), None if c is None else host(c), None if r is None else host(r), 77, 8, 9)
        assert np.array_equal(got[1].cpu().numpy(), qs) and np.array_equal(got[3].cpu().numpy(), qts)
        assert np.array_equal(got[0].cpu().numpy(), q)
        assert np.array_equal(got[2].cpu().numpy(), np.swapaxes(q * 0 + qt, 1, 2))
        # sums of T terms: 32 of each wavefront, 4 of them, the chunks of 128 rows one after another
        d = host(dy).astype(np.float64)
        assert np.all(np.abs(got[4].cpu().numpy() - d.sum(1)) <= (32 + 4 + T / 128 + 1) * 2.0 ** -24 * np.abs(d).sum(1))
        again = lowbit.quantize_grad(a, c, r, seed=77, iter=8, site=9)
        assert all(torch.equal(u, v) for u, v in zip(got, again))


def test_gradients_that_are_not_finite_show():
    dy = normal((1, 140, 530), torch.float32, 24)
    dy[0, 3, 520] = float("inf")
    dy[0, 130, 7] = float("nan")
    q, qs, qt, qts, sums = lowbit.quantize_grad(dy, seed=1, iter=2, site=3)
    assert qs[0].isnan().nonzero().flatten().tolist() == [3, 130] and qts[0].isnan().nonzero().flatten().tolist() == [7, 520]
    assert not sums[0].isfinite()[[7, 520]].any() and int(sums[0].isfinite().sum()) == 528
    fine = torch.ones(140, dtype=torch.bool)
    fine[[3, 130]] = False
    clean = dy.clone()
    clean[0, 3, 520], clean[0, 130, 7] = 0.0, 0.0
    assert torch.equal(q[0, fine], lowbit.quantize_grad(clean, seed=1, iter=2, site=3)[0][0, fine])


# ---- products

def random_codes(shape, seed, low=-127):
    return torch.randint(low, 128, shape, generator=gen(seed), device=DEV, dtype=torch.int32).to(torch.int8)


def held(codes):
    """Rows 16 bytes apart, what is behind them not zero."""
    cols = codes.shape[-1]
    big = torch.full((*codes.shape[:-1], -(-cols // 16) * 16), 55, dtype=torch.int8, device=DEV)
    big[..., :cols] = codes
    return big[..., :cols]


def product_close(got, want, sa, sb, bias, dtype, extra=0):
    """y = fl(fl(fl(sum) sa) sb) + bias, rounded to the type: 3 roundings of the product (and `extra` more), one of the sum, one of the type."""
    term = np.abs(want - (0.0 if bias is None else host(bias).astype(np.float64)))
    allowed = (3.01 + extra) * 2.0 ** -24 * term + 2.0 ** -24 * np.abs(want) + (1 + 2.0 ** -12) * UNIT[dtype] * np.abs(want) + TINIEST[dtype]
    diff = np.abs(host(got).astype(np.float64) - want)
    return bool(np.all(diff <= allowed + 2.0 ** -22 * UNIT[dtype] * term))


SIZES = [(1, 1, 1), (1, 3, 2), (1, 64, 64), (1, 1000, 333), (2, 17, 16), (3, 50, 100), (16, 256, 512), (17, 130, 129), (33, 70, 1000),
         (48, 300, 257), (64, 64, 63), (65, 129, 191), (100, 513, 640), (128, 128, 128), (130, 200, 300), (200, 1025, 77), (257, 255, 1025),
         (300, 520, 2000), (1, 16, 5000), (5, 2049, 4097)]


@pytest.mark.parametrize("size", SIZES)
def test_products(size):
    T, N, K = size
    a, b = random_codes((T, K), 31), random_codes((N, K), 32)
    sa = torch.rand(T, generator=gen(33), device=DEV) * 1e-2
    sb = torch.rand(N, generator=gen(34), device=DEV) * 1e-2
    bias = normal((N,), torch.float32, 35)
    # one call in float64 on the host is exact: sums below 2^53
    for x, w in ((held(a), held(b)), (a, b), (spread(a[None], 0)[0], held(b))):
        for dtype in TYPES:
            for s, c, d in ((sa, sb, bias), (None, None, None), (sa, None, bias), (None, sb, None)):
                if dtype is torch.float16 and (s is None or c is None):
                    continue  # (out of the type's range)
                want = L.product(a.cpu().numpy(), b.cpu().numpy(), *[None if v is None else host(v) for v in (s, c, d)])
                got = lowbit.matmul_i8(x, w, s, c, d, dtype=dtype)
                assert product_close(got, want, s, c, d, dtype), (dtype, s is None, c is None, d is None)


@pytest.mark.parametrize("M,T,N,K", [(1, 5, 7, 9), (2, 33, 65, 100), (3, 1, 64, 64), (4, 130, 70, 257), (2, 64, 256, 512), (5, 16, 16, 16)])
def test_products_of_several_workers(M, T, N, K):
    a = random_codes((M, T, K), 41)
    sa = torch.rand((M, T), generator=gen(42), device=DEV)
    for lead in ((), (M,)):
        b = random_codes((*lead, N, K), 43)
        sb = torch.rand((*lead, N), generator=gen(44), device=DEV)
        bias = normal((N,), torch.float32, 45)
        want = L.product(a.cpu().numpy(), b.cpu().numpy(), host(sa), host(sb), host(bias))
        for x, w in ((held(a), held(b)), (spread(a, 0), b)):
            assert product_close(lowbit.matmul_i8(x, w, sa, sb, bias), want, sa, sb, bias, torch.float32)
        out = torch.full((M, N * T + 40), 7.0, device=DEV)  # where g[M][d] has a layer's gradients
        view = out[:, 11:11 + T * N].view(M, T, N)
        assert lowbit.matmul_i8(held(a), held(b), sa, sb, bias, out=view) is view
        assert product_close(view, want, sa, sb, bias, torch.float32)
        assert (out[:, :11] == 7).all() and (out[:, 11 + T * N:] == 7).all()


@pytest.mark.parametrize("M,T,N,K", [(1, 4100, 4000, 130), (1, 8200, 4200, 257), (3, 2900, 2000, 128), (1, 2100, 3000, 700), (1, 700, 3000, 1111),
                                     (1, 1000, 1000, 513), (4, 300, 700, 64), (1, 2048, 2048, 140000)])
def test_products_of_many_tiles(M, T, N, K):
    """Every kind of tile, whole and not, several for a workgroup, with and without what goes back through dropout."""
    say(f"layer calls: product of {M} x {T} x {N} x {K} codes")
    a, b = random_codes((M, T, K), 46), random_codes((N, K) if M == 1 else (M, N, K), 47)
    sa, sb = torch.rand((M, T), generator=gen(48), device=DEV) * 1e-3, torch.rand(b.shape[:-1], generator=gen(49), device=DEV) * 1e-3
    bias = normal((N,), torch.float32, 50)
    want = torch.stack([a[m].double() @ (b if M == 1 else b[m]).double().t() for m in range(M)])  # (whole numbers below 2^53)
    want = (want * sa[..., None].double() * (sb if M == 1 else sb[:, None, :]).double()).cpu().numpy()
    for dtype in TYPES:
        got = lowbit.matmul_i8(held(a), held(b), sa, sb, bias, dtype=dtype)
        assert product_close(got, want + host(bias).astype(np.float64), sa, sb, bias, dtype), dtype
        x = normal((M, T, N), dtype, 51)
        d = lowbit.Drop(2, 3, 4, 0.25, True)
        keep = torch.from_numpy(L.kept(2, 3, 4, 0.25, (M, T, N))).to(DEV) & ~(x <= 0)
        got = lowbit.matmul_i8(held(a), held(b), sa, sb, dtype=dtype, drop=d, x=x)
        assert not got[~keep].any()
        assert product_close(got, np.where(keep.cpu().numpy(), want * float(L.over_keep(0.25)), 0.0), sa, sb, None, dtype, extra=1), dtype


@pytest.mark.parametrize("M,T,N,K", [(1, 17, 8300, 200), (1, 33, 300, 9000), (1, 64, 16400, 130), (1, 60, 33000, 70), (1, 129, 8200, 1000), (1, 16, 100, 16500),
                                     (2, 40, 5000, 1003), (1, 49, 4100, 333), (1, 5, 8200, 300), (3, 30, 2730, 520)])
def test_products_of_few_rows(M, T, N, K):
    """The kernel for few rows, one tile of channels and two, and the tiles that take over from it."""
    test_products_of_many_tiles(M, T, N, K)


@pytest.mark.parametrize("T,N,K", [(2, 3, 140000), (1, 40, 300001), (130, 70, 131072), (20, 257, 65537), (300, 300, 20000)])
def test_deep_products(T, N, K):
    """All codes at the end of the range: the sum leaves 32 bits."""
    a, b = torch.full((T, K), -128, dtype=torch.int8, device=DEV), torch.full((N, K), -128, dtype=torch.int8, device=DEV)
    b[0] = 127
    want = np.full((T, N), 128.0 * 128 * K)
    want[:, 0] = -128.0 * 127 * K
    got = lowbit.matmul_i8(held(a), held(b))
    assert product_close(got[None], want[None], None, None, None, torch.float32)
    a, b = random_codes((T, K), 51), random_codes((N, K), 52)
    want = (a.double() @ b.double().t()).cpu().numpy()
    assert product_close(lowbit.matmul_i8(held(a), held(b))[None], want[None], None, None, None, torch.float32)


@pytest.mark.parametrize("M,T,N,K", [(1, 9, 30, 40), (2, 33, 66, 100), (3, 130, 257, 64), (2, 1, 1024, 512), (1, 64, 1000, 2000)])
@pytest.mark.parametrize("dtype", TYPES)
def test_products_that_go_back_through_dropout(M, T, N, K, dtype):
    a, b = random_codes((M, T, K), 61), random_codes((N, K), 62)
    sa = torch.rand((M, T), generator=gen(63), device=DEV) * 1e-3
    x = normal((M, T, N), dtype, 64)
    for p, relu in ((0.1, True), (0.5, False), (0.0, True)):
        d = lowbit.Drop(6, 7, 8, p, relu)
        keep = L.kept(6, 7, 8, p, (M, T, N))
        if relu:
            keep = keep & ~(host(x) <= 0)
        want = np.where(keep, L.product(a.cpu().numpy(), b.cpu().numpy(), host(sa)) * float(L.over_keep(p)), 0.0)
        for u, w, z in ((held(a), held(b), x), (a, spread(b[None], 0)[0], spread(x, 0))):
            got = lowbit.matmul_i8(u, w, sa, dtype=dtype, drop=d, x=z if relu else None)
            assert product_close(got, want, sa, None, None, dtype, extra=1)
            assert not got[torch.from_numpy(~keep).to(DEV)].any()


# ---- the layer

@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("M,T,K,N", [(1, 1, 64, 96), (2, 33, 70, 100), (1, 1, 1000, 513), (3, 140, 257, 300), (2, 128, 256, 384)])
def test_linear_and_its_gradient(M, T, K, N, dtype):
    x, dy = normal((M, T, K), dtype, 71), normal((M, T, N), dtype, 72, 1e-2)
    w = lowbit.weight(normal((N, K), torch.float32, 73, K ** -0.5))
    bias = normal((N,), torch.float32, 74)
    qw, sw = w.q.cpu().numpy(), host(w.scale)
    assert np.array_equal(w.qt.cpu().numpy(), qw.T)
    for p, relu in ((0.0, False), (0.2, True)):
        drop = lowbit.Drop(1, 2, 3, p, relu)
        keep = L.kept(1, 2, 3, p, (M, T, K))
        q, s = L.codes(L.dropped(host(x), keep, p, relu), 2)
        y, saved = lowbit.linear(x, w, bias, drop, keep=True)
        assert product_close(y, L.product(q, qw, s[..., 0], sw, host(bias)), None, None, bias, dtype)
        assert torch.equal(lowbit.linear(x, w, bias, drop), y)
        dx, dw, db = lowbit.linear_grad(dy, saved, w, seed=4, iter=5, site=6)
        r, rs, c, cs = L.grad_codes(host(dy), sw, s[..., 0], 4, 5, 6)
        passed = keep & ~(host(x) <= 0) if relu else keep
        assert product_close(dx, np.where(passed, L.product(r, qw.T, rs) * float(L.over_keep(p)), 0.0), None, None, None, dtype, extra=1)
        assert product_close(dw, L.product(np.swapaxes(c, 1, 2), np.swapaxes(q, 1, 2), cs), None, None, None, torch.float32)
        # and against the derivative itself: a drawn code is less than a step off
        exact = np.where(passed, L.product(host(dy).astype(np.float64) * sw, qw.T) * float(L.over_keep(p)), 0.0)
        step = rs[..., None] * np.abs(qw.astype(np.float64)).sum(0) * float(L.over_keep(p))
        assert np.all(np.abs(host(dx) - exact) <= step * (1 + 1e-5) + 2 * UNIT[dtype] * np.abs(exact) + step * 2 * UNIT[dtype] + TINIEST[dtype])
        exact = np.swapaxes(host(dy).astype(np.float64) * s, 1, 2) @ q.astype(np.float64)
        assert np.all(np.abs(host(dw) - exact) <= cs[..., None] * np.abs(q.astype(np.float64)).sum(1)[:, None, :] * (1 + 1e-5) + 1e-30)
        assert np.all(np.abs(host(db) - host(dy).astype(np.float64).sum(1)) <= (40 + T / 128) * 2.0 ** -24 * np.abs(host(dy)).astype(np.float64).sum(1))


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("M,T", [(1, 1), (1, 2), (1, 3), (1, 5), (1, 8), (1, 9), (3, 1), (2, 7)])
@pytest.mark.parametrize("K,N", [(1, 5), (7, 16), (8, 33), (100, 50), (128, 1000), (1000, 513), (1025, 40), (4096, 2050), (5000, 130), (20000, 60), (45000, 20)])
def test_few_rows_in_one_call_are_the_two_calls(M, T, K, N, dtype):
    x = normal((M, T, K), dtype, 78)
    w = lowbit.weight(normal((N, K), torch.float32, 79), turned=False)
    bias = normal((N,), torch.float32, 80)
    if T > 2:
        x[0, 1] = 0.0
        x[0, 2, K // 2] = float("inf")
    q, s = lowbit.quantize_rows(x)
    for a in (x, spread(x, 0)):
        for b in (bias, None):
            want = lowbit.matmul_i8(q, w.q, s, w.scale, b, dtype=dtype)
            got = lowbit.linear(a, w, b)
            assert same(got, want.cpu())
            if M == 1:
                assert same(lowbit.linear(a[0], w, b), want[0].cpu())


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("M,T", [(2, 1), (4, 1), (2, 2), (1, 4), (8, 1), (3, 4)])
@pytest.mark.parametrize("K,N", [(8, 16), (100, 50), (1000, 9000), (4100, 130)])
def test_few_rows_of_several_workers(M, T, K, N, dtype):
    x = normal((M, T, K), dtype, 81)
    x[-1, 0] = 0.0
    one = lowbit.weight(normal((N, K), torch.float32, 82), turned=False)
    own = lowbit.weight(normal((M, N, K), torch.float32, 83), turned=False)
    bias = normal((N,), torch.float32, 84)
    for a in (x, spread(x, 0), x[:1].expand(M, T, K)):
        q, s = lowbit.quantize_rows(a)
        for w in (one, own):
            want = lowbit.matmul_i8(q, w.q, s, w.scale, bias, dtype=dtype)
            assert same(lowbit.linear(a, w, bias), want.cpu())
            each = [lowbit.linear(a[m], lowbit.Weight(w.q[m], w.scale[m], None) if w is own else w, bias) for m in range(M)]
            assert same(torch.stack(each), want.cpu())


def test_one_worker_without_a_leading_dimension_is_the_same():
    x, dy = normal((1, 37, 130), torch.bfloat16, 75), normal((1, 37, 65), torch.bfloat16, 76)
    w = lowbit.weight(normal((65, 130), torch.float32, 77))
    drop = lowbit.Drop(1, 2, 3, 0.1, True)
    y3, s3 = lowbit.linear(x, w, None, drop, keep=True)
    y2, s2 = lowbit.linear(x[0], w, None, drop, keep=True)
    assert torch.equal(y3[0], y2)
    for u, v in zip(lowbit.linear_grad(dy, s3, w, seed=1, iter=1, site=1), lowbit.linear_grad(dy[0], s2, w, seed=1, iter=1, site=1)):
        assert torch.equal(u[0], v)


def test_the_gradients_average_to_the_derivative():
    x, dy = normal((2, 20, 30), torch.float32, 81), normal((2, 20, 24), torch.float32, 82)
    w = lowbit.weight(normal((24, 30), torch.float32, 83))
    y, saved = lowbit.linear(x, w, keep=True)
    n, dx, dw = 400, torch.zeros((2, 20, 30), device=DEV, dtype=torch.float64), torch.zeros((2, 24, 30), device=DEV, dtype=torch.float64)
    for it in range(n):
        a, b, _ = lowbit.linear_grad(dy, saved, w, seed=9, iter=it, site=0)
        dx += a
        dw += b
    qw, qx = w.q.double(), saved.qt.double().transpose(1, 2)
    exact_x = (dy.double() * w.scale) @ qw
    exact_w = ((dy.double() * saved.scale[..., None]).transpose(1, 2)) @ qx
    # each term's variance is at most a quarter of a step squared: 6 deviations of the mean
    step_x = (dy.abs() * w.scale).amax(2, keepdim=True) / 127
    step_w = (dy.abs() * saved.scale[..., None]).amax(1)[..., None] / 127
    dev_x = step_x * 0.5 * (qw ** 2).sum(0).sqrt() / n ** 0.5
    dev_w = step_w * 0.5 * (qx ** 2).sum(1).sqrt()[:, None, :] / n ** 0.5
    assert ((dx / n - exact_x).abs() <= 6 * dev_x + 1e-4 * step_x * qw.abs().sum(0)).all()
    assert ((dw / n - exact_w).abs() <= 6 * dev_w + 1e-4 * step_w * qx.abs().sum(1)[:, None, :]).all()


# ---- where the calls run

def test_calls_are_ordered_on_the_current_stream_and_replay_from_a_graph():
    side = torch.cuda.Stream(device=DEV)
    x, dy = normal((2, 130, 257), torch.bfloat16, 91), normal((2, 130, 96), torch.bfloat16, 92)
    w = lowbit.weight(normal((96, 257), torch.float32, 93))
    drop = lowbit.Drop(1, 2, 3, 0.1, True)

    def step(x, dy):
        y, saved = lowbit.linear(x, w, None, drop, keep=True)
        return (y, *lowbit.linear_grad(dy, saved, w, seed=1, iter=2, site=3), lowbit.dropout(x, drop, x), lowbit.dropout_grad(x, drop, x))

    want = step(x, dy)
    other = step(-x, dy)
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        x2, dy2 = x.clone(), dy.clone()
        assert all(torch.equal(u, v) for u, v in zip(step(x2, dy2), want))
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=side):
            held_out = step(x2, dy2)
        for k in range(3):
            say(f"layer calls: graph replay {k}")
            for t in held_out:
                t.zero_()
            x2.copy_(x if k != 1 else -x)
            assert torch.equal(step(x, dy)[0], want[0])
            torch.cuda.synchronize()
            graph.replay()
            torch.cuda.synchronize()
            assert all(torch.equal(u, v) for u, v in zip(held_out, want if k != 1 else other)), f"replay {k}"


def test_calls_through_ctypes_are_the_same(monkeypatch):
    x, dy = normal((2, 37, 90), torch.bfloat16, 98), normal((2, 37, 50), torch.bfloat16, 99)
    w = lowbit.weight(normal((50, 90), torch.float32, 100))
    bias = normal((50,), torch.float32, 101)
    drop = lowbit.Drop(1, 2, 3, 0.1, True)

    def everything():
        y, saved = lowbit.linear(x, w, bias, drop, keep=True)
        out = torch.zeros((2, 50, 90), device=DEV)
        return (y, *lowbit.linear_grad(dy, saved, w, seed=1, iter=2, site=3, out=out), out, lowbit.linear(x, w, bias), lowbit.linear(x[0, :3], w),
                lowbit.dropout(x, drop, x), lowbit.dropout_grad(x, drop, x), *lowbit.quantize_rows(x, drop, True),
                *lowbit.quantize_grad(dy, w.scale, seed=4, iter=5, site=6))

    want = everything()
    plain = lowbit.Drop(1, 2, 3, 0.0)
    zero = lowbit.dropout(x, plain), lowbit.dropout(x, plain._replace(p=0, relu=0)), lowbit.dropout(x, (1, 2, 3, 0.0, False))
    assert torch.equal(zero[0], x) and torch.equal(zero[1], x) and torch.equal(zero[2], x)
    for name in ("_layer", "_linear", "_linear_grad"):
        assert getattr(B, name) is not B._through_ctypes  # (built here)
        monkeypatch.setattr(B, name, B._through_ctypes)
    assert all(torch.equal(u, v) for u, v in zip(everything(), want))


def test_strides_that_pass_32_bits():
    rows, cols, ld = 5, 300, 1 << 30
    say("layer calls: rows 2^30 elements apart")
    far = torch.empty((rows - 1) * ld + 512, dtype=torch.int8, device=DEV)
    q = far.as_strided((rows, cols), (ld, 1))
    a, b = random_codes((rows, cols), 95), random_codes((70, cols), 96)
    q.copy_(a)
    want = lowbit.matmul_i8(a, b)
    assert torch.equal(lowbit.matmul_i8(q, b), want) and torch.equal(lowbit.matmul_i8(b, q), want.t())
    wide = torch.empty((rows - 1) * ld + 512, dtype=torch.bfloat16, device=DEV)
    x = wide.as_strided((rows, cols), (ld, 1))
    x.copy_(normal((rows, cols), torch.bfloat16, 97))
    d = lowbit.Drop(1, 2, 3, 0.5, True)
    near = x.contiguous()
    assert torch.equal(lowbit.dropout(x, d, x), lowbit.dropout(near, d, near))
    assert all(torch.equal(u, v) for u, v in zip(lowbit.quantize_rows(x, d, True), lowbit.quantize_rows(near, d, True)))
    assert all(torch.equal(u, v) for u, v in zip(lowbit.quantize_grad(x, seed=1, iter=1, site=1), lowbit.quantize_grad(near, seed=1, iter=1, site=1)))
    lowbit.dropout_grad(near, d, near, out=x)
    assert torch.equal(x, lowbit.dropout_grad(near, d, near))


def test_refusals():
    f, i = torch.zeros((4, 6), device=DEV), torch.zeros((4, 6), dtype=torch.int8, device=DEV)
    d = lowbit.Drop(1, 2, 3, 0.5)
    with pytest.raises(TypeError):
        lowbit.dropout(f.t(), d)
    with pytest.raises(TypeError):
        lowbit.dropout(f.double(), d)
    with pytest.raises(ValueError):
        lowbit.dropout(f[0], d)
    with pytest.raises(B.TngError):
        lowbit.dropout(f, d._replace(p=1.0))
    with pytest.raises(B.TngError):
        lowbit.dropout(f, d, torch.zeros((4, 5), device=DEV))
    with pytest.raises(B.TngError):
        lowbit.dropout_grad(f, d._replace(relu=True))
    with pytest.raises(TypeError):
        lowbit.matmul_i8(f, i)
    with pytest.raises(B.TngError):
        lowbit.matmul_i8(i, i[:, :5])
    with pytest.raises(ValueError):
        lowbit.matmul_i8(i, i, torch.zeros(5, device=DEV))
    with pytest.raises(TypeError):
        lowbit.matmul_i8(i, i, torch.zeros(4, device=DEV, dtype=torch.float64))
    with pytest.raises(ValueError):
        lowbit.matmul_i8(i, i, out=torch.zeros((4, 5), device=DEV))
    with pytest.raises(TypeError):
        lowbit.matmul_i8(i, i.cpu())
    with pytest.raises(ValueError):
        lowbit.linear_grad(f, None, lowbit.weight(f, turned=False), seed=0, iter=0, site=0)
