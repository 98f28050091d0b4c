"""Host-side checks of the layer calls that need no GPU: what they refuse, before anything is enqueued, and what they size."""
import ctypes

import pytest
import torch

from paper_1901_08227_amd import binding as B
from paper_1901_08227_amd import lowbit

P = 0x100000  # a fake device address: no call below reaches a launch


def mat(rows=4, cols=8, type=B.TYPE_F32, workers=1, ld=None, pitch=None, data=P):
    ld = cols if ld is None else ld
    return B.TngMatrix(data, type, workers, rows, cols, ld, rows * ld if pitch is None else pitch)


def drop(p=0.5, relu=0, site=0):
    return B.TngDrop(1, 2, site, p, relu)


def test_structs_match_the_header_layout():
    assert ctypes.sizeof(B.TngMatrix) == 48 and B.TngMatrix.rows.offset == 16 and B.TngMatrix.pitch.offset == 40
    assert ctypes.sizeof(B.TngDrop) == 24 and B.TngDrop.p.offset == 16 and B.TngDrop.relu.offset == 20


BAD = [dict(type=7), dict(type=-1), dict(workers=0), dict(workers=70000), dict(data=None), dict(data=P + 2), dict(ld=7), dict(ld=1 << 41),
       dict(workers=2, pitch=31), dict(rows=1 << 34), dict(rows=1 << 20, cols=1 << 20)]


@pytest.mark.parametrize("kw", BAD)
def test_matrices_that_are_refused(kw):
    L = B.lib()
    bad, ok = mat(**kw), mat(workers=kw.get("workers", 1) if kw.get("workers") == 2 else 1)
    for x, r, y in ((bad, None, ok), (ok, bad, ok), (ok, None, bad)):
        assert L.tng_dropout(None, drop(), x, r, y) == B.TNG_ERR_INVALID_ARG
    for dy, dx in ((bad, ok), (ok, bad)):
        assert L.tng_dropout_grad(None, drop(), None, dy, dx) == B.TNG_ERR_INVALID_ARG
    assert L.tng_dropout_grad(None, drop(relu=1), bad, ok, ok) == B.TNG_ERR_INVALID_ARG
    assert L.tng_quantize_rows(None, None, bad, mat(type=B.TYPE_I8), P, None) == B.TNG_ERR_INVALID_ARG


def test_dropout_refusals():
    L = B.lib()
    ok = mat()
    for d in (drop(p=1.0), drop(p=-0.1), drop(p=float("nan")), drop(site=1 << 24), drop(relu=2), None):
        assert L.tng_dropout(None, d, ok, None, ok) == B.TNG_ERR_INVALID_ARG
        assert L.tng_dropout_grad(None, d, ok, ok, ok) == B.TNG_ERR_INVALID_ARG
    for other in (mat(rows=5), mat(cols=7), mat(type=B.TYPE_BF16), mat(workers=2), None):
        assert L.tng_dropout(None, drop(), ok, None, other) == B.TNG_ERR_INVALID_ARG
        assert L.tng_dropout_grad(None, drop(relu=1), other, ok, ok) == B.TNG_ERR_INVALID_ARG
    assert L.tng_dropout(None, drop(), ok, mat(rows=5), ok) == B.TNG_ERR_INVALID_ARG
    assert L.tng_dropout(None, drop(), mat(type=B.TYPE_I8), None, mat(type=B.TYPE_I8)) == B.TNG_ERR_INVALID_ARG
    # a broadcast input is none for an output
    assert L.tng_dropout(None, drop(), ok, None, mat(ld=0)) == B.TNG_ERR_INVALID_ARG
    assert L.tng_dropout(None, drop(), mat(workers=2), None, mat(workers=2, pitch=0)) == B.TNG_ERR_INVALID_ARG
    # nothing to write
    assert L.tng_dropout(None, drop(), mat(rows=0, data=None), None, mat(rows=0, data=None)) == B.TNG_OK


def test_quantize_refusals():
    L = B.lib()
    x, q, qt = mat(), mat(type=B.TYPE_I8), mat(rows=8, cols=4, type=B.TYPE_I8)
    assert L.tng_quantize_rows(None, None, x, q, None, None) == B.TNG_ERR_INVALID_ARG
    assert L.tng_quantize_rows(None, None, x, q, P + 1, None) == B.TNG_ERR_INVALID_ARG
    assert L.tng_quantize_rows(None, None, x, mat(), P, None) == B.TNG_ERR_INVALID_ARG
    assert L.tng_quantize_rows(None, None, x, q, P, q) == B.TNG_ERR_INVALID_ARG
    assert L.tng_quantize_rows(None, drop(p=1.0), x, q, P, None) == B.TNG_ERR_INVALID_ARG
    assert L.tng_quantize_rows(None, None, q, q, P, None) == B.TNG_ERR_INVALID_ARG
    big = (1 << 22) + 1
    assert L.tng_quantize_rows(None, None, mat(rows=big), mat(rows=big, type=B.TYPE_I8), P, None) == B.TNG_ERR_INVALID_ARG
    assert L.tng_quantize_rows(None, None, mat(rows=0, data=None), mat(rows=0, type=B.TYPE_I8, data=None), None, None) == B.TNG_OK

    need = L.tng_quantize_grad_bytes(x)
    assert need >= 4 * (4 + 8) and L.tng_quantize_grad_bytes(None) == 0 and L.tng_quantize_grad_bytes(mat(rows=big)) == 0

    def grad(key=drop(), dy=x, cs=None, rs=None, q=q, qs=P, qt=qt, qts=P, sums=P, ws=P, size=need):
        return L.tng_quantize_grad(None, key, dy, cs, rs, q, qs, qt, qts, sums, ws, size)

    for kw in (dict(key=None), dict(dy=None), dict(dy=q), dict(q=x), dict(qt=q), dict(qt=None), dict(qs=None), dict(qts=None),
               dict(cs=P + 2), dict(rs=P + 1), dict(sums=P + 3)):
        assert grad(**kw) == B.TNG_ERR_INVALID_ARG, kw
    for kw in (dict(ws=None), dict(ws=P + 16), dict(size=need - 1)):
        assert grad(**kw) == B.TNG_ERR_WORKSPACE, kw


def test_product_refusals():
    L = B.lib()
    a, b, y = mat(4, 8, B.TYPE_I8), mat(6, 8, B.TYPE_I8), mat(4, 6)
    need = L.tng_matmul_i8_bytes(a, b, y)
    assert need > 0

    def call(a=a, sa=None, b=b, sb=None, bias=None, d=None, x=None, y=y, ws=P, size=need):
        return L.tng_matmul_i8(None, a, sa, b, sb, bias, d, x, y, ws, size)

    bad = [dict(a=None), dict(b=None), dict(y=None), dict(a=mat(4, 8)), dict(b=mat(6, 7, B.TYPE_I8)), dict(y=mat(4, 5)), dict(y=mat(5, 6)),
           dict(y=mat(4, 6, B.TYPE_I8)), dict(y=mat(4, 6, workers=2)), dict(b=mat(6, 8, B.TYPE_I8, workers=2)), dict(sa=P + 1),
           dict(sb=P + 2), dict(bias=P + 3), dict(d=drop(p=1.0)), dict(d=drop(relu=1)), dict(d=drop(relu=1), x=mat(4, 5)),
           dict(d=drop(relu=1), x=mat(4, 6, B.TYPE_F16)), dict(y=mat(4, 6, ld=0))]
    for kw in bad:
        assert call(**kw) == B.TNG_ERR_INVALID_ARG, kw
        if set(kw) <= {"a", "b", "y"}:
            assert L.tng_matmul_i8_bytes(kw.get("a", a), kw.get("b", b), kw.get("y", y)) == 0
    for kw in (dict(ws=None), dict(ws=P + 8), dict(size=need - 1)):
        assert call(**kw) == B.TNG_ERR_WORKSPACE, kw
    big = (1 << 22) + 1
    assert call(a=mat(4, big, B.TYPE_I8), b=mat(6, big, B.TYPE_I8)) == B.TNG_ERR_INVALID_ARG
    assert call(a=mat(0, 8, B.TYPE_I8, data=None), y=mat(0, 6, data=None), ws=None, size=0) == B.TNG_OK


def test_linear_refusals():
    L = B.lib()
    x, b, y = mat(4, 8, B.TYPE_F16), mat(6, 8, B.TYPE_I8), mat(4, 6, B.TYPE_F16)
    need = L.tng_linear_i8_bytes(x, b, y)
    assert need >= 4 * 16 + 4 * 4

    def call(d=None, x=x, b=b, sb=None, bias=None, y=y, ws=P, size=need):
        return L.tng_linear_i8(None, d, x, b, sb, bias, y, ws, size)

    for kw in (dict(x=None), dict(b=None), dict(y=None), dict(x=mat(4, 8)), dict(x=mat(4, 8, B.TYPE_I8)), dict(x=mat(4, 7, B.TYPE_F16)), dict(b=x),
               dict(y=mat(4, 5, B.TYPE_F16)), dict(y=mat(4, 6)), dict(d=drop(p=1.0)), dict(sb=P + 1), dict(bias=P + 2)):
        assert call(**kw) == B.TNG_ERR_INVALID_ARG, kw
        if set(kw) <= {"x", "b", "y"}:
            assert L.tng_linear_i8_bytes(kw.get("x", x), kw.get("b", b), kw.get("y", y)) == 0
    for kw in (dict(ws=None), dict(ws=P + 8), dict(size=need - 1)):
        assert call(**kw) == B.TNG_ERR_WORKSPACE, kw
    assert call(x=mat(0, 8, B.TYPE_F16, data=None), y=mat(0, 6, B.TYPE_F16, data=None), ws=None, size=0) == B.TNG_OK


def test_a_product_of_many_pieces_sizes_their_sums():
    L = B.lib()
    a, b, y = mat(100, 1 << 18, B.TYPE_I8), mat(6, 1 << 18, B.TYPE_I8), mat(100, 6)
    assert L.tng_matmul_i8_bytes(a, b, y) >= 4 * 100 * 6 * 4


def test_host_tensors_are_refused():
    x, d = torch.zeros(2, 3), lowbit.Drop(0, 0, 0)
    for call in (lambda: lowbit.dropout(x, d), lambda: lowbit.dropout_grad(x, d), lambda: lowbit.quantize_rows(x),
                 lambda: lowbit.matmul_i8(x.to(torch.int8), x.to(torch.int8)),
                 lambda: lowbit.quantize_grad(x, seed=0, iter=0, site=0)):
        with pytest.raises(TypeError):
            call()
