"""Host-side checks of the orthogonalised update that need no GPU: what is refused, before anything is enqueued, and what is sized."""
import ctypes

import pytest
import torch

from paper_1901_08227_amd import binding as B
from paper_1901_08227_amd import update
from test_lowbit_abi import BAD, P, mat


def plan(coefficients=(update.QUINTIC,) * 5, eps=1e-7, scale=1.0, steps=None):
    flat = [v for step in coefficients for v in step]
    return B.TngOrthogonal((ctypes.c_float * max(1, len(flat)))(*flat), len(coefficients) if steps is None else steps, eps, scale)


def test_struct_matches_the_header_layout():
    assert ctypes.sizeof(B.TngOrthogonal) == 24 and B.TngOrthogonal.steps.offset == 8 and B.TngOrthogonal.scale.offset == 16


@pytest.mark.parametrize("kw", BAD)
def test_matrices_that_are_refused(kw):
    L = B.lib()
    bad, ok = mat(**kw), mat(workers=2 if kw.get("workers") == 2 else 1)
    for x, y in ((bad, ok), (ok, bad)):
        assert L.tng_orthogonalize(None, x, plan(), y, P, 1 << 40) == B.TNG_ERR_INVALID_ARG


def test_refusals():
    L = B.lib()
    x = mat(6, 9)
    need = L.tng_orthogonalize_bytes(x)
    assert need > 0

    def call(x=x, p=None, y=x, ws=P, size=need):
        return L.tng_orthogonalize(None, x, plan() if p is None else p, y, ws, size)

    nan, inf = float("nan"), float("inf")
    bad = [dict(x=None), dict(y=None), dict(x=mat(6, 9, B.TYPE_I8)), dict(x=mat(6, 9, B.TYPE_I64)), dict(y=mat(6, 9, B.TYPE_I8)), dict(y=mat(9, 6)), dict(y=mat(6, 9, workers=2)),
           dict(y=mat(6, 9, ld=0)), dict(p=plan(steps=0)), dict(p=plan(((1.5, -0.5, 0.0),) * 65)), dict(p=plan(eps=0.0)), dict(p=plan(eps=1e-40)),
           dict(p=plan(eps=nan)), dict(p=plan(eps=inf)), dict(p=plan(scale=nan)), dict(p=plan(scale=inf)), dict(p=plan(((1.5, nan, 0.0),))),
           dict(p=plan(((1.5, -0.5, inf),))), dict(p=B.TngOrthogonal(None, 1, 1e-7, 1.0)), dict(x=mat(65537, 1), y=mat(65537, 1)),
           dict(x=mat(1, 65537), y=mat(1, 65537))]
    for kw in bad:
        assert call(**kw) == B.TNG_ERR_INVALID_ARG, kw
    assert L.tng_orthogonalize(None, x, None, x, P, need) == B.TNG_ERR_INVALID_ARG
    for a in (None, mat(65537, 1), mat(1, 65537), mat(6, 9, B.TYPE_I8)):
        assert L.tng_orthogonalize_bytes(a) == 0
    for kw in (dict(ws=None), dict(ws=P + 64), dict(size=need - 1)):
        assert call(**kw) == B.TNG_ERR_WORKSPACE, kw
    for shape in ((0, 9), (9, 0)):
        none = mat(*shape, data=None)
        assert call(x=none, y=none, ws=None, size=0) == B.TNG_OK


@pytest.mark.parametrize("coefficients,fits", [
    ((update.QUINTIC,) * 64, True), (((1.5, -0.5, 0.0),) * 64, True), (((1.875, -1.25, 0.375),) * 64, True), (((1.0, 0.0, 0.0),) * 64, True),
    (((1.9, 0.0, 0.0),), True), (((2.0, 0.0, 0.0),), False), (((1.9, 0.0, 0.0),) * 2, False), (((-1.9, 0.0, 0.0),), True), (((8.5, -20.0, 12.0),), False),
    (((7.0, -16.0, 10.0),), True), (((7.0, -16.0, 10.0),) * 2, False), (((0.0, 0.0, 2.0),), False), (((7.0, 0.0, -7.0),), False), (((3e38, 3e38, 3e38),), False)])
def test_coefficients_that_leave_the_range_are_refused(coefficients, fits):
    # by the definition: the largest values over a grid of singular values
    import numpy as np
    top, want = 1.0, True
    for a, b, c in coefficients:
        s = np.linspace(0, top, 100001)
        p = a + b * s ** 2 + c * s ** 4
        want = want and np.max(np.abs(p)) < 7.9 and np.max(np.abs(s * p)) < 1.97
        top = min(np.max(np.abs(s * p)), 10.0)
    assert want == fits
    x = mat(6, 9)
    got = B.lib().tng_orthogonalize(None, x, plan(coefficients), x, None, 0)
    assert got == (B.TNG_ERR_WORKSPACE if fits else B.TNG_ERR_UNSUPPORTED)


def test_host_tensors_and_wrong_coefficients_are_refused():
    with pytest.raises(TypeError):
        update.orthogonalize(torch.zeros(2, 3))
