"""The oracle of norms and embeddings: its gradients against differences of its own functions."""
import numpy as np

from oracle import token_oracle as O


def differences(f, x, step=1e-6):
    out = np.zeros_like(x)
    for i in np.ndindex(*x.shape):
        a, b = x.copy(), x.copy()
        a[i] += step
        b[i] -= step
        out[i] = (f(a) - f(b)) / (2 * step)
    return out


def test_norm_gradient_is_that_of_the_norm():
    rng = np.random.default_rng(1)
    h, w, dy, r = rng.normal(size=(3, 7)), rng.normal(size=7), rng.normal(size=(3, 7)), rng.normal(size=(3, 7))
    for eps in (1e-6, 0.5):
        dx, dw = O.rms_norm_grad(dy, h, w, eps, r)
        f = lambda v: np.sum(dy * O.rms_norm(v, w, eps)) + np.sum(r * v)  # noqa: E731
        # central differences of step d are off by d^2 / 6 of a third derivative, and 2^-53 / d of the sum: 1e-9 covers both
        assert np.max(np.abs(dx - differences(f, h))) < 1e-8
        assert np.max(np.abs(dw - differences(lambda v: np.sum(dy * O.rms_norm(h, v, eps)), w))) < 1e-8


def test_large_rows_and_zeros():
    y = O.rms_norm(np.array([[3e38, 4e38], [0.0, 0.0]]), None, 1e-6)
    assert np.allclose(y, [[3 / np.sqrt(12.5), 4 / np.sqrt(12.5)], [0, 0]], rtol=1e-15)


def test_embedding_gradient_counts_a_token_as_often_as_it_comes():
    ids = np.array([2, 0, 2, -1, 5, 2])
    dy = np.arange(12.0).reshape(6, 2)
    out, size = O.embed_grad(ids, dy, 4, -2.0)
    want = np.zeros((4, 2))
    for t, v in enumerate(ids):
        if 0 <= v < 4:
            want[v] += -2.0 * dy[t]
    assert np.array_equal(out, want) and np.array_equal(size, np.abs(want))
