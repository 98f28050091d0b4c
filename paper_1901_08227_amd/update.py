"""The update of matrices by what the server has decoded (include/tng.h on torch tensors): gradients orthogonalised before the step.

Tensors are [rows, cols], or [M, rows, cols] for M matrices, as in lowbit; nothing is recorded by autograd.  After a decoded average vbar

    w -= lr * orthogonalize(vbar_of_w, scale=max(1, rows / cols) ** 0.5)

where Context.step would take w -= lr vbar.
"""
from __future__ import annotations

import ctypes

import torch

from . import binding as B
from . import lowbit

QUINTIC = (3.4445, -4.775, 2.0315)  # a, b, c of the Muon optimiser: five steps bring singular values between 0.003 and 1 near 1 (0.68 to 1.21)


def orthogonalize(x, coefficients=(QUINTIC,) * 5, eps=1e-7, scale=1.0, out=None):
    """scale times x with its singular values brought near 1: X = x / (||x|| + eps), then for each (a, b, c) of the coefficients
    X = (a + b G + c G G) X with G = X X^T.  Each matrix by itself; the result is of x's type, or of out's."""
    device = x.device
    if device.type != "cuda":
        raise TypeError("x: expected a CUDA tensor")
    if any(len(step) != 3 for step in coefficients):
        raise ValueError("coefficients: expected (a, b, c) for each step")
    flat = [float(v) for step in coefficients for v in step]
    if out is None:
        got = lowbit._make("tng_orthogonalize", device, "mjow", x, (*flat, float(eps), float(scale)))
        if got is not None:
            return got
        out = torch.empty(x.shape, dtype=x.dtype, device=device)
    else:
        out = lowbit._out(out, x.shape, out.dtype, device)
    plan = B.TngOrthogonal((ctypes.c_float * len(flat))(*flat), len(coefficients), float(eps), float(scale))
    a, y = lowbit._matrix(x, lowbit._TYPES, "x"), lowbit._matrix(out, lowbit._TYPES, "out")
    L = B.lib()
    with torch.cuda.device(device):
        scratch = torch.empty(L.tng_orthogonalize_bytes(a), dtype=torch.uint8, device=device)
        B._check(L.tng_orthogonalize(lowbit._stream(device), a, plan, y, scratch.data_ptr(), scratch.numel()), "tng_orthogonalize")
    return out
