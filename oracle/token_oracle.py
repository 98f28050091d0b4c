"""Embedding tables and root-mean-square norms in binary64, from their formulas (numpy; test infrastructure only)."""
import numpy as np


def mean_square(h):
    """Along the last axis (binary64 holds the square of every binary32 number)."""
    return np.mean(h ** 2, axis=-1, keepdims=True)


def rms_norm(h, weight, eps):
    h = h.astype(np.float64)
    w = 1.0 if weight is None else weight.astype(np.float64)
    return h / np.sqrt(mean_square(h) + eps) * w


def rms_norm_grad(dy, h, weight, eps, dresidual=None):
    """(dx, dw): dw over the last but one axis."""
    dy, h = dy.astype(np.float64), h.astype(np.float64)
    g = dy if weight is None else dy * weight.astype(np.float64)
    s = 1.0 / np.sqrt(mean_square(h) + eps)
    unit = h * s
    dx = s * (g - unit * np.mean(g * unit, axis=-1, keepdims=True))
    if dresidual is not None:
        dx = dx + dresidual.astype(np.float64)
    return dx, np.sum(dy * unit, axis=-2)


def embed_grad(ids, dy, vocabulary, scale):
    """One worker's: ids [T], dy [T, cols].  (The gradient, and the sums of the magnitudes that it is made of.)"""
    out, size = np.zeros((vocabulary, dy.shape[1])), np.zeros((vocabulary, dy.shape[1]))
    inside = (ids >= 0) & (ids < vocabulary)
    np.add.at(out, ids[inside], dy[inside].astype(np.float64))
    np.add.at(size, ids[inside], np.abs(dy[inside].astype(np.float64)))
    return out * scale, size * abs(scale)
