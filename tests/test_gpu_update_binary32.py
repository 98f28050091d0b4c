"""Orthogonalised updates of every kind of kernel, held to what binary32 itself makes of them.

The bound that test_gpu_update.py follows through the steps grows by the largest slope each time, to a few per cent of the result at five; here the measure is
the error of the same steps in binary32 (elementary products of the library, on the GPU), four times that and three roundings of 22 bits.  That this line passes
no operand which loses its lower half anywhere is shown in test_oracle_update_bits.py."""
import pytest
import torch

from gpu_util import say
from oracle import update_oracle as O
from paper_1901_08227_amd import update
from test_gpu_lowbit import normal
from test_gpu_token_network import make
from test_gpu_update import CUBIC, QUINTIC, SHAPES, step_in

pytestmark = pytest.mark.gpu

STRIPS = [(3, 5, 1100), (2, 20, 3000), (1, 32, 8192), (1, 40, 2500), (2, 64, 8000), (1, 70, 1000), (2, 96, 2100), (40, 66, 900), (1, 64, 1024)]
LONG = [(2, 1, 2000), (3, 2, 65536), (2, 3, 4097), (70, 33, 1030), (1, 33, 8193)]
TILES = [(1, 128, 129), (2, 97, 300), (1, 70, 5000), (2, 200, 3000), (3, 500, 2600), (9, 700, 777), (1, 1100, 1030)]


def as_binary32(got, x, coefficients, scale=1.0):
    """One matrix's result against binary64's and binary32's."""
    want, plain = step_in(x.double(), coefficients) * scale, step_in(x, coefficients) * scale
    return O.as_binary32(*(t.double().cpu().numpy() for t in (got, want, plain)))


@pytest.mark.parametrize("coefficients", [QUINTIC[:1], QUINTIC[:2], QUINTIC, CUBIC])
@pytest.mark.parametrize("shape", SHAPES + STRIPS + LONG + TILES)
def test_no_further_off_than_binary32(shape, coefficients):
    say(f"update: {shape}, {len(coefficients)} steps")
    x = normal(shape, torch.float32, 1, 1e-3)
    y = update.orthogonalize(x, coefficients, scale=1.25)
    z = update.orthogonalize(x.transpose(1, 2).contiguous(), coefficients, scale=1.25).transpose(1, 2)
    for k in {0, shape[0] - 1}:
        # (step_in takes the products over the first side: x turned where that is the longer one)
        turned = shape[1] > shape[2]
        a, got = (x[k].t().contiguous(), (y[k].t(), z[k].t())) if turned else (x[k], (y[k], z[k]))
        for g in got:
            assert as_binary32(g, a, coefficients, 1.25)


def test_the_networks_orthogonal_step():
    """The steps of the layers' weights, from the decoded average that the step itself went by."""
    net = make(orthogonal=True, lr=1.0)
    net.w.zero_()  # (weights of zeros: what is left after the step is the step, without a rounding)
    net.g.normal_(generator=torch.Generator(device=net.device).manual_seed(5))
    net.orthogonal_step(0)
    for (w, _), (v, _) in zip(net.layers(net.w), net.layers(net.vbar)):
        scale = max(1.0, w.shape[0] / w.shape[1]) ** 0.5
        wide = w.shape[0] <= w.shape[1]
        a, got = (v, -w) if wide else (v.t(), -w.t())
        assert v.norm() > 0 and as_binary32(got, a.contiguous(), QUINTIC, scale)
    net.close()
