"""The scale of an orthogonalised update: one product in binary32, whatever its size."""
import numpy as np
import pytest
import torch

from gpu_util import DEV
from paper_1901_08227_amd import update
from test_gpu_lowbit import TYPES, normal, same

pytestmark = pytest.mark.gpu


# one launch, strips (wide and tall), tiles, and tiles that several workgroups share
@pytest.mark.parametrize("shape", [(2, 40, 60), (1, 128, 100), (1, 50, 1300), (1, 1300, 50), (2, 300, 500), (1, 500, 300), (1, 120, 3000)])
@pytest.mark.parametrize("scale", [1.25, -3e4, 1e-31, 1e-36, 2.0 ** -126, -1e-37, 1e-42, 1e37, 0.0])
def test_results_are_those_of_a_scale_of_one_times_the_scale(shape, scale):
    x = normal(shape, torch.float32, 80)
    one, got = update.orthogonalize(x), update.orthogonalize(x, scale=scale)
    # a product of two binary32 numbers is exact in binary64, from where it is rounded once
    assert same(got, (one.cpu().double() * float(np.float32(scale))).float())


@pytest.mark.parametrize("dtype", TYPES)
def test_a_small_scale_into_every_type(dtype):
    x = normal((2, 40, 60), torch.float32, 81)
    wide = update.orthogonalize(x, scale=1e-6)
    out = torch.empty(x.shape, dtype=dtype, device=DEV)
    assert same(update.orthogonalize(x, scale=1e-6, out=out), wide.cpu().to(dtype))
