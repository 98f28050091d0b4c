"""The layer calls at the sizes where another kernel takes over, beyond 32 bits, and with something else's bytes behind their rows, against the oracle."""
import numpy as np
import pytest
import torch

from gpu_util import DEV, say
from oracle import lowbit_oracle as L
from oracle import tng_oracle as O
from paper_1901_08227_amd import lowbit
from test_gpu_lowbit import gen, held, host, normal, product_close, random_codes, rounded, same, spread

pytestmark = pytest.mark.gpu


def filled(shape, value, dtype):
    return torch.full(shape, value, dtype=dtype, device=DEV)


# workers, rows, columns.  The kernel that codes takes 128 x 128 tiles in two halves from 1024 of them on; 64 x 128 ones, of which up to 1024
# put the statistics of up to 64 chunks of rows and 32 runs of 512 columns together themselves.
GRADIENTS = [
    ((4, 2048, 2048), torch.bfloat16),  # 1024 tiles
    ((1, 4096, 4096), torch.float32),
    ((8, 1000, 2040), torch.float16),
    ((8, 128, 16384), torch.bfloat16),
    ((3, 1408, 3968), torch.bfloat16),  # 1023
    ((5, 513, 5127), torch.float32),    # 1025
    ((4, 2048, 2176), torch.float16),   # 1088
    ((1, 2048, 4096), torch.bfloat16),  # 1024 tiles of 64 rows, 64 chunks of 32
    ((1, 2049, 4096), torch.float32),   # 1056
    ((1, 1024, 4096), torch.float16),   # 64 chunks of 16
    ((2, 400, 8200), torch.bfloat16),   # 25 chunks, 17 runs of columns
    ((1, 400, 16384), torch.float32),   # 32 runs of columns
    ((1, 400, 16385), torch.bfloat16),  # 33
    ((1, 512, 130), torch.float16),     # 64 chunks of 8
    ((1, 520, 130), torch.float32),     # 65
]


@pytest.mark.parametrize("shape,dtype", GRADIENTS)
def test_codes_of_a_gradient_where_another_kernel_takes_over(shape, dtype):
    M, T, N = shape
    say(f"layer calls: codes of a gradient of {M} x {T} x {N}")
    dy = normal(shape, dtype, 121, 1e-2)
    dy[0, T // 2] = 0.0
    dy[M - 1, :, N - 1] = 0.0
    cs = torch.rand(N, generator=gen(122), device=DEV) + 0.5
    rs = torch.rand((M, T), generator=gen(123), device=DEV) + 0.5
    q, qt = filled(shape, 77, torch.int8), filled((M, N, T), 77, torch.int8)
    qs, qts, sums = (filled(s, -7.0, torch.float32) for s in ((M, T), (M, N), (M, N)))
    lowbit._run("tng_quantize_grad", dy.device, lowbit.Drop(78, 9, 10), dy, cs, rs, q, qs, qt, qts, sums)
    want_q, want_qs, want_qt, want_qts = L.grad_codes(host(dy), host(cs), host(rs), 78, 9, 10)
    assert np.array_equal(qs.cpu().numpy(), want_qs) and np.array_equal(qts.cpu().numpy(), want_qts)
    assert np.array_equal(q.cpu().numpy(), want_q)
    assert np.array_equal(qt.cpu().numpy(), np.swapaxes(want_qt, 1, 2))
    # Additions of a column: a quarter of a chunk's rows, four wavefronts, the chunks.  A chunk has 8, 16, 32 or 64 rows.
    most = max(rows // 4 - 1 + 3 + -(-T // rows) - 1 for rows in (8, 16, 32, 64))
    d = host(dy).astype(np.float64)
    assert np.all(np.abs(sums.cpu().numpy() - d.sum(1)) <= most * 2.0 ** -24 * 1.001 * np.abs(d).sum(1))


# From 1024 rows on a wavefront takes a row and holds 2, 4 or 8 pieces of 512 columns; before, and up to 8192 columns, a workgroup does.
ROWS = [(1, 1024, 513), (2, 520, 1024), (1, 1030, 1025), (3, 400, 2048), (1, 1024, 2049), (1, 1100, 4096), (1, 1024, 4097), (1, 1023, 1024), (2, 511, 4090)]


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16, torch.float16])
@pytest.mark.parametrize("shape", ROWS)
def test_codes_of_rows_that_a_wavefront_holds(shape, dtype):
    say(f"layer calls: codes of {shape[0]} x {shape[1]} x {shape[2]}")
    x = normal(shape, dtype, 131)
    x[0, 5] = 0.0
    for drop in (None, lowbit.Drop(3, 4, 5, 0.25, True)):
        v = host(x)
        if drop is not None:
            v = L.dropped(v, L.kept(3, 4, 5, drop.p, shape), drop.p, drop.relu)
        want, scale = L.codes(v, 2)
        for a in (x, spread(x, 0)):
            q, s, qt = lowbit.quantize_rows(a, drop, turned=True)
            assert np.array_equal(s.cpu().numpy(), scale[..., 0])
            assert np.array_equal(q.cpu().numpy(), want)
            assert np.array_equal(qt.cpu().numpy(), np.swapaxes(want, 1, 2))


# ---- elements beyond the 32 bits of their number

FAR = ((1 << 20) + 5, 4099)
LAST = 40  # of the rows that are compared with the oracle


def last_words(seed, it, site, stream):
    rows, cols = FAR
    return O._draw_words(seed, it, 0, stream | site << 8, (rows - LAST) * cols, LAST * cols).reshape(1, LAST, cols)


@pytest.mark.parametrize("dtype,shape", [(torch.bfloat16, (2, 8200, 4099)), (torch.float16, (1, 16500, 4096)), (torch.float32, (3, 3000, 4001))])
def test_dropout_past_the_caches(dtype, shape):
    """More than 256 MiB of operands; by rows, from operands with gaps, it takes another kernel."""
    M, rows, cols = shape
    say(f"layer calls: dropout of {M} x {rows} x {cols}")
    x, res = normal(shape, dtype, 147), normal(shape, dtype, 148)
    assert 2 * x.numel() * x.element_size() > 256 << 20
    gap = spread(x, 0)
    for relu in (False, True):
        d = lowbit.Drop(5, 6, 7, 0.25, relu)
        words = O._draw_words(5, 6, M - 1, L.STREAM_DROPOUT | 7 << 8, (rows - LAST) * cols, LAST * cols).reshape(LAST, cols)
        keep = (words >> 8) * 2.0 ** -24 >= 0.25
        xe, re = host(x[-1, -LAST:]), host(res[-1, -LAST:])
        for got, by_rows, want in ((lowbit.dropout(x, d), lowbit.dropout(gap, d), L.dropout(xe, keep, 0.25, relu)),
                                   (lowbit.dropout(x, d, res), lowbit.dropout(gap, d, res), L.dropout(xe, keep, 0.25, relu, re)),
                                   (lowbit.dropout_grad(res, d, x), lowbit.dropout_grad(res, d, gap), L.dropout_grad(re, keep, 0.25, relu, xe))):
            assert torch.equal(got, by_rows) and same(got[-1, -LAST:], rounded(want, dtype))


def test_dropout_of_elements_beyond_32_bits():
    rows, cols = FAR
    assert (rows - LAST) * cols >= 1 << 32
    say("layer calls: dropout of 2^32 elements")
    d = lowbit.Drop(5, 6, 7, 0.5, True)
    keep = (last_words(5, 6, 7, L.STREAM_DROPOUT) >> 8) * 2.0 ** -24 >= 0.5
    row = normal((1, cols), torch.bfloat16, 141)
    x = row.expand(rows, cols)              # no gaps where it is written, so by rows
    end = np.repeat(host(row), LAST, 0)[None]
    want = rounded(L.dropout(end, keep, 0.5, True), torch.bfloat16)[0]
    by_rows = lowbit.dropout(x, d)
    assert same(by_rows[-LAST:], want)
    run = x.contiguous()                    # as one run
    assert torch.equal(lowbit.dropout(run, d, out=run), by_rows)
    assert same(lowbit.dropout_grad(by_rows, d, x)[-LAST:], rounded(L.dropout_grad(want[None].float().numpy(), keep, 0.5, True, end), torch.bfloat16)[0])


def test_codes_of_elements_beyond_32_bits():
    rows, cols = FAR
    say("layer calls: codes of 2^32 elements")
    row = normal((1, cols), torch.bfloat16, 142)
    end = np.repeat(host(row), LAST, 0)[None]
    x = row.expand(rows, cols)
    q, s = lowbit.quantize_rows(x, lowbit.Drop(5, 6, 7, 0.5, True))
    want, scale = L.codes(L.dropped(end, (last_words(5, 6, 7, L.STREAM_DROPOUT) >> 8) * 2.0 ** -24 >= 0.5, 0.5, True), 2)
    assert np.array_equal(q[-LAST:].cpu().numpy(), want[0]) and np.array_equal(s[-LAST:].cpu().numpy(), scale[0, :, 0])
    del q
    rs = torch.rand(rows, generator=gen(143), device=DEV) + 0.5
    rs[-LAST // 2] = 2.0                    # so the columns' largest products are in a row that is compared
    q, qs, qt, qts, _ = lowbit.quantize_grad(x, None, rs, seed=8, iter=9, site=10, sums=False)
    w = last_words(8, 9, 10, L.STREAM_ROUNDING)
    want, scale = L.codes(end, 2, w >> 16)
    assert np.array_equal(q[-LAST:].cpu().numpy(), want[0]) and np.array_equal(qs[-LAST:].cpu().numpy(), scale[0, :, 0])
    want, scale = L.codes(end * host(rs)[None, -LAST:, None], 1, w & 0xFFFF)
    assert np.array_equal(qt[:, -LAST:].cpu().numpy(), want[0].T) and np.array_equal(qts.cpu().numpy(), scale[0, 0])


def test_results_beyond_32_bits():
    rows, cols = FAR
    say("layer calls: a product of 2^32 results")
    a, b = random_codes((rows, 16), 144), random_codes((cols, 16), 145)
    x = normal((1, cols), torch.bfloat16, 146).expand(rows, cols)
    d = lowbit.Drop(5, 6, 7, 0.5, True)
    keep = ((last_words(5, 6, 7, L.STREAM_DROPOUT) >> 8) * 2.0 ** -24 >= 0.5) & ~(host(x[-LAST:])[None] <= 0)
    want = np.where(keep, 2.0 * (a[-LAST:].double() @ b.double().t()).cpu().numpy()[None], 0.0)
    y = lowbit.matmul_i8(a, b, dtype=torch.bfloat16, drop=d, x=x)
    assert product_close(y[None, -LAST:], want, None, None, None, torch.bfloat16, extra=1)
    assert not y[-LAST:][torch.from_numpy(~keep[0]).to(DEV)].any()


# ---- what lies behind a row

@pytest.mark.parametrize("M,T,N,K", [(1, 1, 1008, 1000), (1, 1, 40, 7), (1, 1, 513, 20001), (4, 1, 300, 1000), (1, 200, 1, 1000), (3, 100, 1, 77), (1, 1, 1, 130)])
def test_what_lies_behind_a_single_row_does_not_matter(M, T, N, K):
    """A matrix's only row counts as aligned by its address; its last 16 bytes, which are read as a piece, hold something else's codes."""
    a, b = random_codes((M, T, K), 151), random_codes((M, N, K), 152)
    sa, sb = torch.rand((M, T), generator=gen(153), device=DEV), torch.rand((M, N), generator=gen(154), device=DEV)
    want = L.product(a.cpu().numpy(), b.cpu().numpy(), host(sa), host(sb))

    def single(codes, other):
        """[M, 1, K] codes, strides (16 bytes' multiple, K, 1)."""
        big = random_codes((M, -(-K // 16) * 16 + 16), other, -128)
        big[:, :K] = codes[:, 0]
        view = big[:, :K].unsqueeze(1)
        assert view.stride() == (big.shape[1], K, 1)
        return view

    for other in (155, 156):
        u = single(a, other) if T == 1 else held(a)
        v = single(b, other + 2) if N == 1 else held(b)
        assert product_close(lowbit.matmul_i8(u, v, sa, sb), want, sa, sb, None, torch.float32)
        if N == 1:  # and where the rows are coded on the way
            x = normal((M, T, K), torch.float32, 157)
            q, s = lowbit.quantize_rows(x)
            got = [lowbit.linear(x, lowbit.Weight(w, sb)) for w in (v, b)]
            assert torch.equal(*got) and product_close(got[0], L.product(q.cpu().numpy(), b.cpu().numpy(), host(s), host(sb)), s, sb, None, torch.float32)
