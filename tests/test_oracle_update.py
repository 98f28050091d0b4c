"""The oracle of orthogonalised updates: singular values go through the polynomial, singular vectors stay."""
import numpy as np
import pytest

from oracle import update_oracle as O

QUINTIC = ((3.4445, -4.775, 2.0315),) * 5


@pytest.mark.parametrize("shape", [(1, 1), (5, 5), (4, 9), (9, 4)])
@pytest.mark.parametrize("coefficients", [QUINTIC, ((1.5, -0.5, 0.0),) * 3, ((1.875, -1.25, 0.375),)])
def test_singular_values(shape, coefficients):
    x = np.random.default_rng(3).normal(size=shape)
    u, s, v = np.linalg.svd(x, full_matrices=False)
    s = s / (np.linalg.norm(x) + 1e-3)
    for a, b, c in coefficients:
        s = a * s + b * s ** 3 + c * s ** 5
    assert np.allclose(O.orthogonalize(x, coefficients, 1e-3, 2.5), 2.5 * (u * s) @ v, rtol=0, atol=1e-11)


def test_the_bound_of_the_error_holds_for_binary32():
    rng = np.random.default_rng(4)
    x = rng.normal(size=(12, 30))
    want, bound = O.orthogonalize(x, QUINTIC, 1e-7, 1.0, (2.0 ** -24, 0.0, lambda k: (k + 1) * 2.0 ** -24))
    y = (x / (np.linalg.norm(x) + 1e-7)).astype(np.float32)
    for a, b, c in np.float32(QUINTIC):
        g = y @ y.T
        y = (a * np.eye(12, dtype=np.float32) + b * g + c * (g @ g)) @ y
    assert np.linalg.norm(y - want) <= bound
