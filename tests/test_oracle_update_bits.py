"""The line that holds results of the orthogonalised update to binary32's: it passes products of operands of 22 bits, and none that lose the lower 11 of them
anywhere, at any number of steps.  (Mistakes are planted in the oracle; what they would do on the GPU is not run there.)"""
import numpy as np
import pytest

from oracle import update_oracle as O

QUINTIC = ((3.4445, -4.775, 2.0315),) * 5
CUBIC = ((1.5, -0.5, 0.0),) * 3
SHAPES = [(5, 8), (33, 64), (64, 256), (96, 257), (128, 128), (20, 3000), (64, 2000)]
WHOLE = dict(gram=22, square=22, poly=22, apply=22)


def parts(shape, coefficients, seed=1):
    x = np.random.default_rng(seed).normal(size=shape).astype(np.float32)
    return x, O.orthogonalize(x, coefficients, 1e-7, 1.0), O.step_in(x, coefficients, 1e-7).astype(np.float64)


@pytest.mark.parametrize("coefficients", [QUINTIC[:1], QUINTIC[:2], QUINTIC, CUBIC])
@pytest.mark.parametrize("shape", SHAPES)
def test_operands_of_22_bits_pass(shape, coefficients):
    for seed in range(3):
        x, want, plain = parts(shape, coefficients, seed)
        assert O.as_binary32(O.in_bits(x, coefficients, 1e-7, WHOLE), want, plain)


# (A polynomial without c has no G G in it.  In one step of n even rows G is about 1 / n, and 2^-12 of c G G to a is 2^-12 0.6 / n^2, which is below 3 2^-22 from
# 15 rows on: that loss shows from two steps on.)
LOSSES = [(k, part) for k in (QUINTIC[:1], QUINTIC[:2], QUINTIC, CUBIC) for part in WHOLE if part != "square" or k in (QUINTIC[:2], QUINTIC)]


@pytest.mark.parametrize("coefficients,lost", LOSSES)
@pytest.mark.parametrize("shape", SHAPES)
def test_operands_that_lose_their_low_parts_do_not(shape, coefficients, lost):
    x, want, plain = parts(shape, coefficients)
    assert not O.as_binary32(O.in_bits(x, coefficients, 1e-7, WHOLE | {lost: 11}), want, plain)


def test_columns_that_are_left_out_do_not():
    x, want, plain = parts((64, 2000), QUINTIC)
    got = O.in_bits(x, QUINTIC, 1e-7, WHOLE)
    got[:, -1] = 0
    assert not O.as_binary32(got, want, plain)
