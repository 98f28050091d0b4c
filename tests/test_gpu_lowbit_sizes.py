"""The coders at the sizes where another kernel takes over, against the oracle."""
import numpy as np
import pytest
import torch

from gpu_util import DEV, say
from oracle import lowbit_oracle as L
from paper_1901_08227_amd import lowbit
from test_gpu_lowbit import gen, host, normal

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
