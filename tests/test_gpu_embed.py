"""Embedding tables on the GPU: rows bit for bit, gradients against the oracle in binary64.

A gradient's sum of n tokens has at most n - 1 additions and the scale's product: n units of 2^-24 of the sum of the magnitudes."""
import numpy as np
import pytest
import torch

from gpu_util import DEV
from oracle import token_oracle as O
from paper_1901_08227_amd import binding as B
from paper_1901_08227_amd import lowbit
from test_gpu_lowbit import TYPES, gen, host, normal, same, spread

pytestmark = pytest.mark.gpu


def tokens(M, T, V, seed, kind="even", dtype=torch.int64):
    ids = torch.randint(0, max(1, V), (M, T), generator=gen(seed), device=DEV)
    if kind == "skewed":  # most tokens are one or its neighbours, some are outside
        u = torch.rand((M, T), generator=gen(seed + 1), device=DEV)
        ids = torch.where(u < 0.6, min(7, V - 1), ids)
        ids = torch.where(u > 0.9, torch.where(u > 0.95, -1, V), ids)
    elif kind == "one":
        ids.fill_(V - 1)
    elif kind == "none":
        ids.fill_(-5)
    elif kind == "far":
        ids = ids + (1 << (40 if dtype == torch.int64 else 30))
    return ids.to(dtype)


def rows_of(ids, table, scale, dtype):
    """Plain, on the host."""
    ids, table, out = ids.cpu(), table.cpu(), []
    for m in range(ids.shape[0]):
        t = table if table.dim() == 2 else table[m]
        inside = (ids[m] >= 0) & (ids[m] < t.shape[0])
        rows = t[torch.where(inside, ids[m], 0).long()].float() * torch.tensor(scale, dtype=torch.float32) if t.shape[0] else torch.zeros((ids.shape[1], t.shape[1]))
        out.append(torch.where(inside[:, None], rows, 0.0).to(dtype))
    return torch.stack(out)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("of_table", TYPES)
@pytest.mark.parametrize("M,T,V,C", [(1, 1, 1, 1), (2, 3, 5, 7), (3, 50, 11, 8), (2, 33, 300, 129), (1, 700, 40, 1003), (2, 9, 4, 4096)])
def test_rows(M, T, V, C, of_table, dtype):
    table = normal((V, C), of_table, 1)
    for kind, i in (("skewed", torch.int64), ("even", torch.int32), ("none", torch.int32)):
        ids = tokens(M, T, V, 2, kind, i)
        for scale in (1.0, 5.6568542):
            want = rows_of(ids, table, scale, dtype)
            assert same(lowbit.embed(ids, table, scale, dtype), want)
            out = spread(torch.zeros((M, T, C), dtype=dtype, device=DEV), 0)
            wide = spread(table[None], 0)[0]
            assert lowbit.embed(ids, wide, scale, out=out) is out and same(out, want)
    each = normal((M, V, C), of_table, 3)
    assert same(lowbit.embed(ids := tokens(M, T, V, 4), each, 2.0, dtype), rows_of(ids, each, 2.0, dtype))
    assert lowbit.embed(ids, table).dtype == of_table and same(lowbit.embed(ids[0], table), rows_of(ids[:1], table, 1.0, of_table)[0])


GRADS = [(1, 1, 1, 1), (2, 3, 5, 7), (3, 50, 11, 8), (2, 33, 300, 129), (1, 700, 40, 1003), (2, 1024, 16, 40), (1, 1025, 15, 64), (2, 2100, 17, 520), (1, 4096, 33, 24),
         (1, 5000, 3, 72), (2, 8192, 100, 16), (1, 8193, 70000, 9), (1, 30011, 600, 33), (1, 70000, 2, 5)]


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("M,T,V,C", GRADS)
def test_gradient(M, T, V, C, dtype):
    dy = normal((M, T, C), dtype, 5)
    for kind, i in (("skewed", torch.int64), ("even", torch.int32), ("one", torch.int64), ("none", torch.int32), ("far", torch.int64)):
        ids = tokens(M, T, V, 6, kind, i)
        got = lowbit.embed_grad(ids, dy, V, 3.25)
        assert got.shape == (M, V, C) and got.dtype == torch.float32
        for m in range(M):
            n = ids[m].cpu().numpy()
            want, size = O.embed_grad(n, host(dy[m]), V, 3.25)
            count = np.bincount(n[(n >= 0) & (n < V)], minlength=V)[:, None]
            assert np.all(np.abs(got[m].double().cpu().numpy() - want) <= count * 2.0 ** -24 * size), kind
        out = spread(torch.full_like(got, float("nan")), 0)
        assert lowbit.embed_grad(ids, spread(dy, 0), V, 3.25, out=out) is out and torch.equal(out, got)
        assert torch.equal(lowbit.embed_grad(ids, dy, V, 3.25), got)


# the most blocks of sorted tokens that 2^19 make, and the largest tables, whose rows' numbers take 22 and 23 bits
@pytest.mark.parametrize("M,T,V,C", [(1, 1 << 19, 7, 9), (2, 300001, 70000, 5), (1, 5000, (1 << 22) - 1, 3), (2, 200, 1 << 22, 8), (1, 9, 1 << 22, 5)])
def test_gradient_of_many(M, T, V, C):
    test_gradient(M, T, V, C, torch.float32)


def test_gradients_are_written_nowhere_else():
    big = torch.full((3, 20, 50), 7.0, device=DEV)
    ids, dy = tokens(3, 100, 16, 7, "skewed"), normal((3, 100, 33), torch.float32, 8)
    lowbit.embed_grad(ids, dy, 16, out=big[:, 2:18, 9:42])
    assert big[:, :2].eq(7).all() and big[:, 18:].eq(7).all() and big[:, :, :9].eq(7).all() and big[:, :, 42:].eq(7).all()


def test_tokens_with_strides_and_one_worker():
    ids, table = tokens(1, 64, 30, 9)[0], normal((30, 17), torch.bfloat16, 10)
    dy = normal((64, 17), torch.bfloat16, 11)
    want, grad = lowbit.embed(ids, table), lowbit.embed_grad(ids, dy, 30)
    assert want.shape == (64, 17) and grad.shape == (30, 17)
    wide = torch.full((64, 3), -9, device=DEV)
    wide[:, 1] = ids
    assert same(lowbit.embed(wide[:, 1], table), want.cpu()) and torch.equal(lowbit.embed_grad(wide[:, 1], dy, 30), grad)
    # one token, one worker's tokens, that stand for all
    same_ids = ids[5:6].expand(64)
    assert same(lowbit.embed(same_ids, table), lowbit.embed(same_ids.contiguous(), table).cpu())
    assert torch.equal(lowbit.embed_grad(ids.expand(3, 64), dy.expand(3, 64, 17), 30), grad.expand(3, 30, 17))
    with pytest.raises(B.TngError):  # workers that alternate
        lowbit.embed(torch.stack([ids, ids], 1).t(), table)


def test_nothing():
    table, dy = normal((4, 8), torch.float32, 12), torch.empty((2, 0, 8), device=DEV)
    ids = torch.empty((2, 0), dtype=torch.int64, device=DEV)
    assert lowbit.embed(ids, table).shape == (2, 0, 8)
    out = torch.full((2, 4, 8), float("nan"), device=DEV)
    assert lowbit.embed_grad(ids, dy, 4, out=out).eq(0).all()
    assert lowbit.embed(tokens(2, 5, 4, 13), table[:0]).eq(0).all()
    assert lowbit.embed_grad(tokens(2, 5, 4, 13), normal((2, 5, 8), torch.float32, 14), 0).shape == (2, 0, 8)
    assert lowbit.embed(tokens(2, 5, 4, 13), table[:, :0]).shape == (2, 5, 0)
    with pytest.raises(TypeError):
        lowbit.embed(tokens(1, 5, 4, 13).to(torch.int16), table)
    with pytest.raises(ValueError):
        lowbit.embed(tokens(1, 5, 4, 13)[None], table)


def test_what_is_not_finite_stays_in_its_row():
    ids, dy = tokens(1, 3000, 20, 15), normal((1, 3000, 40), torch.float32, 16)
    dy[0, 77, 3] = float("nan")
    dy[0, 1500, 39] = float("inf")
    got, clean = lowbit.embed_grad(ids, dy, 20)[0], lowbit.embed_grad(ids, torch.nan_to_num(dy, 0, 0), 20)[0]
    bad = torch.zeros((20, 40), dtype=torch.bool, device=DEV)
    bad[ids[0, 77], 3] = bad[ids[0, 1500], 39] = True
    assert got[bad].isfinite().logical_not().all() and torch.equal(got[~bad], clean[~bad])


def test_a_table_beyond_32_bits():
    # 2^22 rows of 1056 columns, bfloat16: more than 2^32 elements; tokens at both ends
    V, C = 1 << 22, 1056
    table = torch.zeros((V, C), dtype=torch.bfloat16, device=DEV)
    ids = torch.tensor([0, V - 1, V // 2, V, V - 2, 1], device=DEV)
    table[ids[[0, 1, 2, 4, 5]]] = normal((5, C), torch.bfloat16, 17)
    want = table[ids.clamp(max=V - 1)]
    want[3] = 0
    assert same(lowbit.embed(ids, table), want.cpu())
    del table
    dy = normal((6, C), torch.bfloat16, 18)
    got = lowbit.embed_grad(ids, dy, V)
    assert torch.equal(got[ids[[0, 1, 2, 4, 5]]], dy[[0, 1, 2, 4, 5]].float())
    got[ids[[0, 1, 2, 4, 5]]] = 0
    assert not got.any()


def test_graph_and_another_stream():
    ids, dy, table = tokens(2, 3000, 500, 19, "skewed"), normal((2, 3000, 72), torch.float16, 20), normal((500, 72), torch.float32, 21)
    side, graph = torch.cuda.Stream(), torch.cuda.CUDAGraph()
    want = lowbit.embed(ids, table, 2.0, torch.float16), lowbit.embed_grad(ids, dy, 500, 2.0)
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        got = lowbit.embed(ids, table, 2.0, torch.float16), lowbit.embed_grad(ids, dy, 500, 2.0)
    torch.cuda.current_stream().wait_stream(side)
    assert all(torch.equal(a, b) for a, b in zip(got, want))
    with torch.cuda.graph(graph):
        got = lowbit.embed(ids, table, 2.0, torch.float16), lowbit.embed_grad(ids, dy, 500, 2.0)
    for k in range(3):
        ids.copy_(tokens(2, 3000, 500, 30 + k, "skewed"))
        graph.replay()
        torch.cuda.synchronize()
        want = lowbit.embed(ids, table, 2.0, torch.float16), lowbit.embed_grad(ids, dy, 500, 2.0)
        assert all(torch.equal(a, b) for a, b in zip(got, want))


def test_ctypes_way_is_the_same(monkeypatch):
    ids, dy, table = tokens(2, 300, 50, 22, "skewed"), normal((2, 300, 72), torch.float16, 23), normal((50, 72), torch.float32, 24)
    calls = lambda: (lowbit.embed(ids, table, 2.0, torch.float16), lowbit.embed_grad(ids, dy, 50, 2.0))  # noqa: E731
    want = calls()
    monkeypatch.setattr(B, "_layer", B._through_ctypes)
    assert all(torch.equal(a, b) for a, b in zip(calls(), want))


def test_results_beyond_32_bits_of_no_row_and_of_no_token():
    T, C = 1 << 22, 1100
    out = torch.ones((T, C), dtype=torch.bfloat16, device=DEV)
    table = torch.empty((0, C), dtype=torch.bfloat16, device=DEV)
    assert not lowbit.embed(torch.zeros(T, dtype=torch.int32, device=DEV), table, out=out).any()
    out = torch.ones((T, C), device=DEV)
    assert not lowbit.embed_grad(torch.empty(0, dtype=torch.int64, device=DEV), torch.empty((0, C), device=DEV), T, out=out).any()
