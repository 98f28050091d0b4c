"""Pins of the layer oracle: what its codes, products and gradients have to be whatever the implementation."""
import numpy as np
import pytest

from oracle import lowbit_oracle as L
from oracle import tng_oracle as O


def rng(seed):
    return np.random.default_rng(seed)


def test_nearest_codes_are_within_half_a_step_and_reach_127():
    v = rng(0).normal(size=(3, 5, 301)).astype(np.float32)
    q, s = L.codes(v, 2)
    assert s.shape == (3, 5, 1) and np.array_equal(np.abs(q).max(2), np.full((3, 5), 127))
    assert np.all(np.abs(q * s.astype(np.float64) - v) <= s * (0.5 + 1e-4))


def test_codes_of_rows_that_hold_nothing():
    v = np.zeros((1, 3, 4), dtype=np.float32)
    v[0, 1] = 1e-39                    # below the smallest normal number
    v[0, 2, 0] = O.FLT_MIN
    q, s = L.codes(v, 2)
    assert np.array_equal(s[0, :2, 0], [0, 0]) and not q[0, :2].any() and q[0, 2, 0] == 127 and s[0, 2, 0] > 0
    v[0, 0, 1], v[0, 1, 1] = np.nan, np.inf
    assert np.isnan(L.codes(v, 2)[1][0, :2]).all()


def test_drawn_codes_are_unbiased_by_enumeration_of_every_draw():
    halves = np.arange(1 << 16, dtype=np.uint32)
    for value in (0.3, -0.3, 0.999, -1.0, 1.0, 0.0, 3.7e-5):
        v = np.full((1, 2, 1 << 16), value, dtype=np.float32)
        v[0, 1] = 1.0
        q, s = L.codes(np.swapaxes(v, 1, 2).copy(), 2, np.stack([halves, halves], 1)[None])
        x = float(np.clip(np.float32(value), -1, 1) * np.float32(127))
        mean = q[0, :, 0].astype(np.float64).mean()
        assert abs(mean - x) <= 2.0 ** -16 and abs(np.mean(q[0, :, 0] > np.floor(x)) - L.probability_up(x)) == 0
        assert np.all(np.abs(q) <= 127)


def test_dropout_draws_are_the_generators_and_differ_by_site_worker_and_iteration():
    a = L.kept(7, 3, 1, 0.25, (2, 33, 17))
    assert abs(a.mean() - 0.75) < 5 * np.sqrt(0.25 * 0.75 / a.size)
    assert not np.array_equal(a[0], a[1])
    for other in (L.kept(7, 3, 2, 0.25, a.shape), L.kept(7, 4, 1, 0.25, a.shape), L.kept(8, 3, 1, 0.25, a.shape)):
        assert not np.array_equal(a, other)
    w = L.words(7, 3, 1, L.STREAM_DROPOUT, 2, 33, 17)
    block = O.philox4x32_10(np.uint64(40 // 4), 1, 3, 3 + 256, 7, 0)
    assert w[1].reshape(-1)[41] == block[1]
    assert L.kept(7, 3, 1, 0.0, (1, 2, 3)).all()


def test_dropout_and_its_gradient_against_differences():
    x = rng(1).normal(size=(2, 9, 11))
    x = (np.sign(x) * (np.abs(x) + 0.5)).astype(np.float32)  # away from relu's corner
    keep = L.kept(3, 0, 0, 0.5, x.shape)
    dy = rng(2).normal(size=x.shape).astype(np.float32)
    for with_relu in (False, True):
        h = np.float32(2.0 ** -4)
        up, down = L.dropout(x + h, keep, 0.5, with_relu), L.dropout(x - h, keep, 0.5, with_relu)
        slope = (up.astype(np.float64) - down) / (2 * float(h))
        got = L.dropout_grad(dy, keep, 0.5, with_relu, x)
        # values below 8 scaled by 2 are off by 2^-21 each, twice over 2 h
        assert np.all(np.abs(got - slope * dy) <= 2.0 ** -16 * np.abs(dy))


@pytest.mark.parametrize("M", [1, 3])
def test_gradients_of_the_product_against_differences(M):
    """The derivative of sum(dy y) by the decoded tokens and weights, which linear_grad estimates without bias."""
    g = rng(5)
    T, K, N = 4, 6, 5
    qx, sx = L.codes(g.normal(size=(M, T, K)).astype(np.float32), 2)
    qw, sw = L.codes(g.normal(size=(1, N, K)).astype(np.float32), 2)
    dy = g.normal(size=(M, T, N))
    xs, ws = qx * sx.astype(np.float64), qw[0] * sw[0].astype(np.float64)

    def f(x, w):
        return float(np.sum(dy * (x @ w.T)))

    dx = L.product(dy * sw[0, :, 0], np.ascontiguousarray(qw[0].T))
    dw = np.einsum("mtn,mtk->nk", dy * sx, qx)
    for _ in range(20):
        m, t, k, n = g.integers(M), g.integers(T), g.integers(K), g.integers(N)
        for arr, grad, at in ((xs, dx, (m, t, k)), (ws, dw, (n, k))):
            h = 0.25
            plus, minus = arr.copy(), arr.copy()
            plus[at] += h
            minus[at] -= h
            slope = (f(plus, ws) - f(minus, ws)) / (2 * h) if arr is xs else (f(xs, plus) - f(xs, minus)) / (2 * h)
            assert abs(slope - grad[at]) <= 1e-10 * (1 + abs(slope))


def test_gradient_codes_average_to_the_gradient():
    g = rng(6)
    dy = g.normal(size=(1, 5, 7)).astype(np.float32)
    cs, rs = (0.5 + g.random(7)).astype(np.float32), (0.5 + g.random((1, 5))).astype(np.float32)
    total_r, total_c, n = np.zeros(dy.shape), np.zeros(dy.shape), 400
    for it in range(n):
        q, qs, c, ccs = L.grad_codes(dy, cs, rs, 1, it, 0)
        total_r += q * qs[:, :, None].astype(np.float64)
        total_c += c * ccs[:, None, :].astype(np.float64)
    # a drawn code's variance is at most a quarter of a step squared: 5 deviations of the mean, and the draws' own grid
    assert np.all(np.abs(total_r / n - dy * cs) <= qs[:, :, None] * (2.5 / np.sqrt(n) + 2.0 ** -15))
    assert np.all(np.abs(total_c / n - dy * rs[:, :, None]) <= ccs[:, None, :] * (2.5 / np.sqrt(n) + 2.0 ** -15))
