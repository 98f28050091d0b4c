"""Results that lie where an input begins, and are not that input, are refused without a GPU: what one row's work writes, another's would still read."""
import pytest

from paper_1901_08227_amd import binding as B
from test_lowbit_abi import P, mat
from test_token_abi import ids, num, rms
from test_update_abi import plan

F32, BF16, F16, I8 = B.TYPE_F32, B.TYPE_BF16, B.TYPE_F16, B.TYPE_I8
Q = P + (1 << 20)  # somewhere else
BYTES = 1 << 30

# an input, and a result at its place that is another matrix
OTHERS = [
    (dict(ld=0), dict()),                                   # one row for all
    (dict(ld=8), dict(ld=16)),                              # rows that lie apart otherwise
    (dict(workers=3, pitch=0), dict(workers=3)),            # one matrix for all workers
    (dict(workers=3), dict(workers=3, pitch=64)),           # matrices that lie apart otherwise
    (dict(workers=2, rows=1, pitch=0), dict(workers=2, rows=1)),
]


def calls(x, y, **at):
    """Every call with an input x and a result y of its type and size; the others lie elsewhere."""
    L, there = B.lib(), dict(workers=x.workers, rows=x.rows, cols=x.cols, data=Q)
    other, q = mat(**there), mat(type=I8, **there)
    yield lambda: L.tng_rms_norm(None, x, None, rms(), None, y)
    yield lambda: L.tng_rms_norm(None, other, x, rms(), None, y)
    yield lambda: L.tng_rms_norm(None, x, None, rms(), y, mat(**{**there, "data": Q + 4096}))
    yield lambda: L.tng_rms_norm_codes(None, other, x, rms(), y, q, P, None)
    yield lambda: L.tng_rms_norm_grad(None, x, other, None, rms(), y, None, P, BYTES)
    yield lambda: L.tng_rms_norm_grad(None, other, x, None, rms(), y, None, P, BYTES)
    yield lambda: L.tng_rms_norm_grad(None, other, other, x, rms(), y, None, P, BYTES)
    yield lambda: L.tng_orthogonalize(None, x, plan(), y, P, BYTES)


@pytest.mark.parametrize("x,y", OTHERS)
def test_another_matrix_at_an_inputs_place(x, y):
    for k, call in enumerate(calls(mat(**x), mat(**y))):
        assert call() == B.TNG_ERR_INVALID_ARG, k


def test_the_same_matrix_is_no_other_one():
    """Strides that no index reaches say nothing.  (A workspace that is too small is what is found wrong, behind the places.)"""
    L = B.lib()
    for x, y in ((mat(), mat()), (mat(pitch=0), mat(pitch=99)), (mat(rows=1, ld=0), mat(rows=1, ld=50)), (mat(workers=3), mat(workers=3))):
        assert L.tng_orthogonalize(None, x, plan(), y, P, 0) == B.TNG_ERR_WORKSPACE
        for dy, h, r in ((x, mat(workers=x.workers, rows=x.rows, data=Q), None), (mat(workers=x.workers, rows=x.rows, data=Q), x, x)):
            assert L.tng_rms_norm_grad(None, dy, h, r, rms(), y, None, P, 0) == B.TNG_ERR_WORKSPACE


def test_codes_and_other_types_at_an_inputs_place():
    L = B.lib()
    x, q, qt = mat(), mat(type=I8, data=Q), mat(8, 4, I8, data=Q + 4096)
    for kw in (dict(q=mat(type=I8)), dict(qt=mat(8, 4, I8)), dict(qt=mat(8, 4, I8, data=Q)), dict(r=mat(data=Q)), dict(h=mat(data=Q)), dict(h=mat(data=Q + 4096))):
        a = dict(r=None, h=None, q=q, qt=qt) | kw
        assert L.tng_rms_norm_codes(None, x, a["r"], rms(), a["h"], a["q"], P + 8192, a["qt"]) == B.TNG_ERR_INVALID_ARG, kw
    for a, b in ((F32, BF16), (BF16, F32), (F16, BF16)):
        assert L.tng_orthogonalize(None, mat(type=a), plan(), mat(type=b), P, BYTES) == B.TNG_ERR_INVALID_ARG


def test_rows_of_tokens_at_the_tables_or_the_tokens_place():
    L = B.lib()
    assert L.tng_embed(None, ids(data=Q), mat(16, 8), num(1.0), mat(4, 8)) == B.TNG_ERR_INVALID_ARG
    assert L.tng_embed(None, ids(4), mat(4, 8, data=Q), num(1.0), mat(4, 8)) == B.TNG_ERR_INVALID_ARG
    none = mat(4, 0)
    assert L.tng_embed(None, ids(4), mat(16, 0), num(1.0), none) == B.TNG_OK
