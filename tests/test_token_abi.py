"""Host-side checks of norms and embeddings that need no GPU: what they refuse, before anything is enqueued, and what they size."""
import ctypes

import pytest
import torch

from paper_1901_08227_amd import binding as B
from paper_1901_08227_amd import lowbit
from test_lowbit_abi import BAD, P, mat

I32, I64 = B.TYPE_I32, B.TYPE_I64


def rms(eps=1e-6, weight=P):
    return B.TngRms(weight, eps)


def ids(rows=4, type=I64, workers=1, **kw):
    return mat(rows, 1, type, workers, **kw)


def num(x):
    return ctypes.c_float(x)


def test_struct_matches_the_header_layout():
    assert ctypes.sizeof(B.TngRms) == 16 and B.TngRms.eps.offset == 8


@pytest.mark.parametrize("kw", BAD)
def test_matrices_that_are_refused(kw):
    L = B.lib()
    bad, ok = mat(**kw), mat(workers=2 if kw.get("workers") == 2 else 1)
    q = mat(type=B.TYPE_I8, workers=ok.workers)
    for x, r, h, y in ((bad, None, None, ok), (ok, bad, None, ok), (ok, None, bad, ok), (ok, None, None, bad)):
        assert L.tng_rms_norm(None, x, r, rms(), h, y) == B.TNG_ERR_INVALID_ARG
        if y is ok:
            assert L.tng_rms_norm_codes(None, x, r, rms(), h, q, P, None) == B.TNG_ERR_INVALID_ARG
    for dy, h, r, dx in ((bad, ok, None, ok), (ok, bad, None, ok), (ok, ok, bad, ok), (ok, ok, None, bad)):
        assert L.tng_rms_norm_grad(None, dy, h, r, rms(), dx, P, P, 1 << 30) == B.TNG_ERR_INVALID_ARG


def test_norm_refusals():
    L = B.lib()
    ok, q = mat(), mat(type=B.TYPE_I8)
    need = L.tng_rms_norm_grad_bytes(ok)
    assert need >= 4 * 8 and L.tng_rms_norm_grad_bytes(None) == 0 and L.tng_rms_norm_grad_bytes(q) == 0

    def calls(x=ok, r=None, n=rms(), h=None, y=ok):
        yield lambda: L.tng_rms_norm(None, x, r, n, h, y)
        yield lambda: L.tng_rms_norm_codes(None, x, r, n, h, mat(y.rows, y.cols, B.TYPE_I8, y.workers) if y else None, P, None)
        yield lambda: L.tng_rms_norm_grad(None, x, y, r, n, h or ok, P, P, 1 << 30)

    for n in (None, rms(0.0), rms(-1e-6), rms(float("nan")), rms(float("inf")), rms(1e-40), rms(weight=P + 2)):
        for call in calls(n=n):
            assert call() == B.TNG_ERR_INVALID_ARG
    for other in (mat(rows=5), mat(cols=7), mat(workers=2)):
        for kw in (dict(r=other), dict(h=other), dict(y=other)):
            for call in calls(**kw):
                assert call() == B.TNG_ERR_INVALID_ARG, kw
    half = mat(type=B.TYPE_BF16)
    assert L.tng_rms_norm(None, ok, None, rms(), None, half) == B.TNG_ERR_INVALID_ARG
    assert L.tng_rms_norm(None, ok, half, rms(), None, ok) == B.TNG_ERR_INVALID_ARG
    assert L.tng_rms_norm(None, ok, None, rms(), half, ok) == B.TNG_ERR_INVALID_ARG
    assert L.tng_rms_norm(None, q, None, rms(), None, q) == B.TNG_ERR_INVALID_ARG
    assert L.tng_rms_norm(None, ids(), None, rms(weight=None), None, ids()) == B.TNG_ERR_INVALID_ARG
    # a broadcast input is none for an output
    for out in (mat(ld=0),):
        assert L.tng_rms_norm(None, ok, None, rms(), None, out) == B.TNG_ERR_INVALID_ARG
        assert L.tng_rms_norm(None, ok, None, rms(), out, ok) == B.TNG_ERR_INVALID_ARG
        assert L.tng_rms_norm_grad(None, ok, ok, None, rms(), out, P, P, need) == B.TNG_ERR_INVALID_ARG
    assert L.tng_rms_norm_codes(None, ok, None, rms(), None, q, None, None) == B.TNG_ERR_INVALID_ARG
    assert L.tng_rms_norm_codes(None, ok, None, rms(), None, q, P + 1, None) == B.TNG_ERR_INVALID_ARG
    assert L.tng_rms_norm_codes(None, ok, None, rms(), None, q, P, q) == B.TNG_ERR_INVALID_ARG
    assert L.tng_rms_norm_codes(None, ok, None, rms(), None, ok, P, None) == B.TNG_ERR_INVALID_ARG
    for kw in (dict(dw=P + 1), dict(dx=None), dict(h=None)):
        a = dict(dy=ok, h=ok, dx=ok, dw=P) | kw
        assert L.tng_rms_norm_grad(None, a["dy"], a["h"], None, rms(), a["dx"], a["dw"], P, need) == B.TNG_ERR_INVALID_ARG
    for ws, size in ((None, need), (P + 16, need), (P, need - 1)):
        assert L.tng_rms_norm_grad(None, ok, ok, None, rms(), ok, P, ws, size) == B.TNG_ERR_WORKSPACE
    big = (1 << 22) + 1
    assert L.tng_rms_norm(None, mat(rows=big), None, rms(), None, mat(rows=big)) == B.TNG_ERR_INVALID_ARG
    assert L.tng_rms_norm_grad_bytes(mat(rows=big)) == 0
    # nothing to write
    none = mat(rows=0, data=None)
    assert L.tng_rms_norm(None, none, None, rms(), None, none) == B.TNG_OK
    assert L.tng_rms_norm(None, mat(cols=0, data=None), None, rms(), None, mat(cols=0, data=None)) == B.TNG_OK
    assert L.tng_rms_norm_codes(None, none, None, rms(), None, mat(rows=0, type=B.TYPE_I8, data=None), None, None) == B.TNG_OK
    assert L.tng_rms_norm_grad(None, none, none, None, rms(), none, None, None, 0) == B.TNG_OK


def test_embedding_refusals():
    L = B.lib()
    t, y, i = mat(16, 8), mat(4, 8, B.TYPE_BF16), ids()

    def call(ids=i, table=t, scale=None, y=y):
        return L.tng_embed(None, ids, table, scale, y)

    bad = [dict(ids=None), dict(table=None), dict(y=None), dict(ids=mat(4, 1)), dict(ids=ids(5)), dict(ids=mat(4, 2, I64)), dict(ids=ids(workers=2)),
           dict(ids=ids(data=P + 4)), dict(ids=ids(type=6)), dict(ids=ids(data=None)), dict(table=mat(16, 7)), dict(table=mat(16, 8, B.TYPE_I8)),
           dict(table=mat(16, 8, workers=2)), dict(table=mat((1 << 22) + 1, 8)), dict(table=mat(16, 8, ld=7)), dict(y=mat(4, 8, B.TYPE_I8)),
           dict(y=mat(4, 8, ld=0)), dict(scale=num(float("nan"))), dict(scale=num(float("inf")))]
    for kw in bad:
        assert call(**kw) == B.TNG_ERR_INVALID_ARG, kw
    assert call(ids=ids(0, data=None), y=mat(0, 8, data=None)) == B.TNG_OK
    assert call(table=mat(16, 0, data=None), y=mat(4, 0, data=None)) == B.TNG_OK


def test_embedding_gradient_refusals():
    L = B.lib()
    i, dy, dt = ids(), mat(4, 8, B.TYPE_F16), mat(16, 8)
    need = L.tng_embed_grad_bytes(i, dy, dt)
    assert need > 0

    def call(ids=i, dy=dy, scale=None, dt=dt, ws=P, size=need):
        return L.tng_embed_grad(None, ids, dy, scale, dt, ws, size)

    bad = [dict(ids=None), dict(dy=None), dict(dt=None), dict(ids=mat(4, 1)), dict(ids=ids(5)), dict(ids=ids(workers=2)), dict(dy=mat(4, 8, B.TYPE_I8)),
           dict(dy=mat(4, 7)), dict(dt=mat(16, 8, B.TYPE_F16)), dict(dt=mat(16, 8, workers=2)), dict(dt=mat(16, 8, ld=0)), dict(dt=mat((1 << 22) + 1, 8))]
    for kw in bad:
        assert call(**kw) == B.TNG_ERR_INVALID_ARG, kw
        assert L.tng_embed_grad_bytes(kw.get("ids", i), kw.get("dy", dy), kw.get("dt", dt)) == 0
    assert call(scale=num(float("inf"))) == B.TNG_ERR_INVALID_ARG
    for kw in (dict(ws=None), dict(ws=P + 8), dict(size=need - 1)):
        assert call(**kw) == B.TNG_ERR_WORKSPACE, kw
    assert call(dt=mat(0, 8, data=None), ws=None, size=0) == B.TNG_OK


def test_host_tensors_and_wrong_shapes_are_refused():
    x, i = torch.zeros(2, 3), torch.zeros(2, dtype=torch.int64)
    for call in (lambda: lowbit.rms_norm(x), lambda: lowbit.rms_norm(x, residual=x), lambda: lowbit.rms_norm_codes(x), lambda: lowbit.rms_norm_grad(x, x),
                 lambda: lowbit.embed(i, x), lambda: lowbit.embed_grad(i, x, 5)):
        with pytest.raises(TypeError):
            call()
    with pytest.raises(ValueError):
        lowbit.rms_norm(x, residual=x, out=torch.zeros(3, 3))
    with pytest.raises(ValueError):
        lowbit.embed_grad(i, x, 5, out=torch.zeros(4, 3))


def test_two_results_in_one_place_and_an_eps_beside_which_no_square_counts():
    L = B.lib()
    ok, other = mat(), B.TngMatrix(P + 4096, *[getattr(mat(), f) for f, _ in B.TngMatrix._fields_[1:]])
    assert L.tng_rms_norm(None, ok, None, rms(), other, other) == B.TNG_ERR_INVALID_ARG
    assert L.tng_rms_norm(None, ok, None, rms(2.0 ** 65), None, other) == B.TNG_ERR_INVALID_ARG
    none = mat(rows=0)
    assert L.tng_rms_norm(None, none, None, rms(2.0 ** 64), none, none) == B.TNG_OK
