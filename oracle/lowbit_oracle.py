"""Numpy oracle of the layer calls: dropout by counter, 8-bit codes of rows and gradients, products of codes.

TEST INFRASTRUCTURE ONLY.  What decides a code or a kept element is IEEE binary32 with one rounding per written operation (numpy
float32 ufuncs); sums and everything that follows from the codes is float64.  All arrays are [M, rows, cols].
"""
from __future__ import annotations

import math

import numpy as np

from . import tng_oracle as O

F32 = np.float32
STREAM_DROPOUT = 3
STREAM_ROUNDING = 4


def words(seed, it, site, stream, M, rows, cols):
    """The draw of every element, uint32[M, rows, cols]."""
    return np.stack([O._draw_words(seed, it, m, stream | site << 8, 0, rows * cols).reshape(rows, cols) for m in range(M)])


def kept(seed, it, site, p, shape):
    if p == 0:
        return np.ones(shape, dtype=bool)
    return (words(seed, it, site, STREAM_DROPOUT, *shape) >> 8) * 2.0 ** -24 >= float(F32(p))


def over_keep(p):
    return F32(1.0 / (1.0 - float(F32(p))))


def relu(x):
    return np.where(x < 0, F32(0), x)


def dropped(x, keep, p, with_relu):
    """float32: keep f(x) / (1 - p)."""
    with np.errstate(all="ignore"):
        return np.where(keep, (relu(x) if with_relu else x) * over_keep(p), F32(0))


def dropout(x, keep, p, with_relu, residual=None):
    y = dropped(x, keep, p, with_relu)
    return y if residual is None else residual + y


def dropout_grad(dy, keep, p, with_relu, x=None):
    if with_relu:
        keep = keep & ~(x <= 0)
    with np.errstate(all="ignore"):
        return np.where(keep, dy * over_keep(p), F32(0))


def codes(v, axis, halves=None):
    """(codes, scales): along `axis`, to nearest or by the 16-bit draws."""
    assert v.dtype == np.float32
    with np.errstate(all="ignore"):
        r = np.max(np.abs(v), axis=axis, keepdims=True) if v.shape[axis] else np.zeros_like(np.sum(v, axis=axis, keepdims=True))
        r = np.where(r < O.FLT_MIN, F32(0), r)
        inv = np.where(r > 0, F32(1) / r, F32(0))
        x = np.clip(v * inv, F32(-1), F32(1)) * F32(127)
        if halves is None:
            q = np.rint(x)
        else:
            low = np.floor(x)
            q = low + (halves.astype(F32) * F32(2.0 ** -16) < x - low)
        step = np.where(np.isfinite(r), r / F32(127), F32(np.nan))
        return np.where(np.isfinite(r), q, 0).astype(np.int8), step.astype(F32)


def grad_codes(dy, col_scale, row_scale, seed, it, site):
    """(row codes, their scales [M, rows], column codes [M, rows, cols], their scales [M, cols])."""
    w = words(seed, it, site, STREAM_ROUNDING, *dy.shape)
    with np.errstate(all="ignore"):
        a = dy if col_scale is None else dy * col_scale[None, None, :]
        b = dy if row_scale is None else dy * row_scale[:, :, None]
    q, qs = codes(a, 2, w >> 16)
    c, cs = codes(b, 1, w & 0xFFFF)
    return q, qs[:, :, 0], c, cs[:, 0, :]


def product(a, b, a_scale=None, b_scale=None, bias=None):
    """float64 [M, rows, channels]; b [channels, depth] or [M, channels, depth]."""
    y = a.astype(np.float64) @ np.swapaxes(b.astype(np.float64), -1, -2)
    if a_scale is not None:
        y = y * a_scale.astype(np.float64)[..., None]
    if b_scale is not None:
        y = y * b_scale.astype(np.float64)[..., None, :]
    return y if bias is None else y + bias.astype(np.float64)


def probability_up(x):
    """P(code = floor(x) + 1): the draws u = 0, 2^-16, ... below the fraction."""
    f = np.float64(x) - math.floor(x)
    return math.ceil(f * 2 ** 16) / 2 ** 16
