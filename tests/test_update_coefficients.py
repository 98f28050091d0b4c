"""Coefficients of an orthogonalised update that are no triples, refused without a GPU."""
import pytest
import torch

from paper_1901_08227_amd import update


class OnGpu:
    """What orthogonalize asks a tensor before it looks at the coefficients."""
    device = torch.device("cuda:0")


# as many numbers as triples have, of too few, too many, an odd number of steps
@pytest.mark.parametrize("coefficients", [
    ((1.5, -0.5), (0.0, 1.5, -0.5, 0.0)), ((1.5, -0.5, 0.0, 1.5), (-0.5, 0.0)), ((1.5, -0.5, 0.0), (1.5,), (-0.5, 0.0, 1.5, -0.5, 0.0)),
    ((), (1.5, -0.5, 0.0, 1.5, -0.5, 0.0)), ((1.5, -0.5),), ((1.5, -0.5, 0.0, 0.0),), [(1.5, -0.5, 0.0), [2.0, 1.0]]])
def test_steps_of_other_than_three_numbers_are_refused(coefficients):
    with pytest.raises(ValueError, match=r"\(a, b, c\)"):
        update.orthogonalize(OnGpu(), coefficients)
