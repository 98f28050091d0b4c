"""What the layer calls' Python side hands to the library where 32 bits do not hold an argument (no GPU needed)."""
import pytest
import torch

from paper_1901_08227_amd import binding as B
from paper_1901_08227_amd import build, lowbit


def refused(drop, matrix=B.TngMatrix(None, B.TYPE_F32, 1, 0, 1, 1, 0)):
    """Whether the library refuses them; nothing is ever written: there are no rows."""
    status = B.lib().tng_dropout(None, drop, matrix, None, matrix)
    assert status in (B.TNG_OK, B.TNG_ERR_INVALID_ARG)
    return status == B.TNG_ERR_INVALID_ARG


@pytest.mark.parametrize("site,bad", [(0, False), ((1 << 24) - 1, False), (1 << 24, True), (-1, True), ((1 << 32) - 1, True), (1 << 32, True),
                                      ((1 << 32) + 3, True), (-(1 << 32) + 3, True), (1 << 80, True)])
def test_sites_do_not_wrap(site, bad):
    assert refused(lowbit._drop(lowbit.Drop(1, 2, site, 0.5))) == bad


class OnTheGpu(torch.Tensor):
    """A tensor of the host that says otherwise."""
    is_cuda = True


@pytest.mark.parametrize("workers,bad", [(1, False), (65535, False), (65536, True), ((1 << 32) + 1, True)])
def test_numbers_of_workers_do_not_wrap(workers, bad):
    x = torch.zeros((1, 0, 1)).as_subclass(OnTheGpu).expand(workers, 0, 1)
    matrix = lowbit._matrix(x, lowbit._TYPES, "x")
    matrix.pitch = 0  # (of no elements)
    assert refused(lowbit._drop(lowbit.Drop(1, 2, 3, 0.5)), matrix) == bad


def test_without_a_native_function_that_fits_layer_calls_go_through_ctypes(monkeypatch, tmp_path):
    names = ("call", "layer", "linear", "linear_grad")
    B.lib()
    built = [getattr(B, "_" + name) for name in names]
    assert B._through_ctypes not in built and len(set(built)) == 4  # (built here)

    def loaded():
        """The four as the library's first use would have them."""
        with monkeypatch.context() as mp:
            for name in ("_lib", "_address", *("_" + name for name in names)):
                mp.setattr(B, name, None)
            B.lib()
            return [getattr(B, "_" + name) for name in names]

    assert loaded() == built
    with monkeypatch.context() as mp:  # built for another torch
        mp.setattr(build, "call_target", lambda: "torch 1.0, cpython-27")
        assert loaded() == [B._through_ctypes] * 4
    with monkeypatch.context() as mp:  # no library
        mp.setattr(B, "CALL_PATH", str(tmp_path / "tng_call.so"))
        assert loaded() == [B._through_ctypes] * 4
        (tmp_path / "tng_call.so").write_text("not a library")
        assert loaded() == [B._through_ctypes] * 4
    assert loaded() == built
