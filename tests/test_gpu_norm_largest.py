"""Norms of rows of the largest numbers that binary32 and bfloat16 hold, in long rows: the sum of their squares, taken down, has to stay in binary32 whatever
the rows' length.

Tolerances as in test_gpu_norm.py.  A row's factor s is down to 2^-128 here, a subnormal number: its last place is 2^-149, a rounding half of that, 2^-22 = 4 U of s."""
import numpy as np
import pytest
import torch

from gpu_util import DEV
from oracle import token_oracle as O
from paper_1901_08227_amd import lowbit
from test_gpu_lowbit import TYPES, host, normal, same
from test_gpu_norm import HALF_STEP, S, U, near, weights

pytestmark = pytest.mark.gpu

LOW = S + 4 * U
COLS = [1, 5, 300, 1000, 1500, 4096, 5000, 7000, 10000, 20011, 30000, 40003]


def largest(cols, dtype, seed=90):
    """Rows between a half and all of the largest number, and such a number in every, and in one column of small ones; a row of ordinary numbers."""
    top = torch.finfo(dtype).max
    gen = torch.Generator(device=DEV)
    gen.manual_seed(seed)
    part = 0.5 + 0.5 * torch.rand((1, 5, cols), generator=gen, device=DEV, dtype=torch.float64)
    sign = torch.where(torch.rand(part.shape, generator=gen, device=DEV) < 0.5, -1.0, 1.0)
    h = (part * sign * top).to(dtype)
    h[0, 1] = top
    h[0, 2] = normal((cols,), dtype, seed + 1)
    h[0, 2, cols // 2] = -top
    h[0, 3] = normal((cols,), dtype, seed + 2)
    assert h.isfinite().all()
    return h


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("cols", COLS)
def test_norm_and_codes(cols, dtype):
    h, w = largest(cols, dtype), weights(cols)
    want = O.rms_norm(host(h), host(w), 1e-5)
    y = lowbit.rms_norm(h, w, eps=1e-5)
    # y = (h s) w: of small h among the largest ones h s is a subnormal number too, off by half of 2^-149 and by w times that as a factor of y
    assert y.isfinite().all() and near(y, want, (LOW + 2 * U) * np.abs(want) + 2.0 ** -150 * np.abs(host(w).astype(np.float64)), dtype)
    # through a residual too, which is all of h
    z, kept = lowbit.rms_norm(torch.zeros_like(h), w, residual=h, eps=1e-5)
    assert same(kept, h.cpu()) and same(z, y.cpu())
    n = lowbit.rms_norm_codes(h, w, eps=1e-5)
    scale = np.abs(want).max(-1) / 127
    assert np.all(np.abs(n.scale.double().cpu().numpy() - scale) <= (LOW + 4 * U) * scale)
    # a code is the nearest whole number to y / scale, or of what is next to a border the other one
    off = np.abs(n.q.double().cpu().numpy() - want / scale[..., None])
    assert np.all(off <= 0.5 + 127 * 2 * (LOW + 8 * U))


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("cols", COLS)
def test_gradient(cols, dtype):
    h, dy, w = largest(cols, dtype), normal((1, 5, cols), dtype, 93), weights(cols)
    dx, dw = lowbit.rms_norm_grad(dy, h, w, eps=1e-5)
    a = [host(t).astype(np.float64) for t in (dy, h, w)]
    want, want_dw = O.rms_norm_grad(a[0], a[1], a[2], 1e-5)
    s = 1 / np.sqrt(O.mean_square(a[1]) + 1e-5)
    unit, g = np.abs(a[1] * s), np.abs(a[0] * a[2])
    along = np.mean(g * unit, -1, keepdims=True)
    # as in test_gpu_norm.py; the row's gradient is a subnormal number itself, of which a product and a rounding to the type are off by half of 2^-149 and of the type's last place
    error = (LOW + 4 * U) * s * g + (75 * U + 3 * LOW + 6 * U) * s * unit * along + 2 * U * np.abs(want) + 2.0 ** -149
    assert dx.isfinite().all() and near(dx, want, error, dtype)
    size = np.sum(np.abs(a[0]) * unit, -2)
    assert np.all(np.abs(dw.double().cpu().numpy() - want_dw) <= (LOW + 9 * U) * size + 5 * 2.0 ** -149)


def test_the_longest_row():
    h = torch.full((1, 1 << 22), torch.finfo(torch.float32).max, device=DEV)
    y = lowbit.rms_norm(h)
    # all alike: y is 1, but for s' rounding, the sum's (of 4096 squares one after another, and of 1024 lanes) and the root's
    assert (y.double() - 1).abs().max().item() <= (4 + 4096 / 2 + 20) * U
    dx, _ = lowbit.rms_norm_grad(torch.ones_like(h), h)
    assert dx.isfinite().all()
    assert HALF_STEP[torch.float32] == U and TYPES[0] == torch.float32
