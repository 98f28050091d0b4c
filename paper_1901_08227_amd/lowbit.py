"""Linear layers of libtng's simulated workers in 8-bit codes, and dropout whose mask is never stored (the layer calls of
include/tng.h on torch tensors).

Tensors are [rows, cols] for one worker or [M, rows, cols] for M of them, float32, bfloat16 or float16, on the GPU, with contiguous
rows; other strides are free.  Everything runs in the library's kernels on the current stream of the tensors' device; results and
scratch come from torch's allocator.  A training step of a layer is

    y, saved = linear(x, weight, bias, drop, keep=True)
    dx, dw, db = linear_grad(dy, saved, weight, seed=..., iter=..., site=...)

with dw and db of every worker, as the coder of the gradients takes them (out= puts them where g[M][d] has them).
"""
from __future__ import annotations

import ctypes
from typing import NamedTuple, Optional

import torch

from . import binding as B

_TYPES = {torch.float32: B.TYPE_F32, torch.bfloat16: B.TYPE_BF16, torch.float16: B.TYPE_F16}


class Drop(NamedTuple):
    """What stands in front of a layer: f(x) = x or relu(x), each element dropped with probability p, the others divided by
    1 - p.  The draws are those of (seed, iter, site, worker, element)."""
    seed: int
    iter: int
    site: int
    p: float = 0.0
    relu: bool = False


class Weight(NamedTuple):
    """Codes of a layer's weights [channels, depth], one scale for each channel; qt: the same codes turned, [depth, channels],
    which the backward pass reads."""
    q: torch.Tensor
    scale: torch.Tensor
    qt: Optional[torch.Tensor] = None


class Saved(NamedTuple):
    """What the backward pass of a layer reads again of its forward pass."""
    x: Optional[torch.Tensor]  # only where a relu's gradient needs it
    drop: Optional[Drop]
    scale: torch.Tensor        # of the tokens' codes, [M, rows]
    qt: torch.Tensor           # the tokens' codes turned, [M, depth, rows]


def _matrix(t, dtypes, name):
    """(tng_matrix, M, rows, cols) of a tensor."""
    if not isinstance(t, torch.Tensor) or not t.is_cuda:
        raise TypeError(f"{name}: expected a CUDA tensor")
    kind = dtypes.get(t.dtype)
    if kind is None:
        raise TypeError(f"{name}: {t.dtype} is not one of {', '.join(map(str, dtypes))}")
    shape, stride = t.shape, t.stride()
    if len(shape) == 2:
        workers, pitch = 1, 0
    elif len(shape) == 3:
        workers, pitch = shape[0], stride[0]
    else:
        raise ValueError(f"{name}: expected [rows, cols] or [M, rows, cols], got {tuple(shape)}")
    if stride[-1] != 1 and shape[-1] > 1:
        raise TypeError(f"{name}: rows have to be contiguous")
    return B.TngMatrix(t.data_ptr(), kind, workers, shape[-2], shape[-1], stride[-2], pitch)


_I8 = {torch.int8: B.TYPE_I8}


def _vector(t, shape, name, device):
    """Address of a contiguous float32 tensor of that shape (None: no address)."""
    if t is None:
        return None
    if not isinstance(t, torch.Tensor) or t.device != device or t.dtype != torch.float32 or not t.is_contiguous():
        raise TypeError(f"{name}: expected contiguous float32 on {device}")
    if t.numel() != shape:
        raise ValueError(f"{name}: needs {shape} elements, has {t.numel()}")
    return t.data_ptr()


def _same_device(device, *tensors):
    for t in tensors:
        if t is not None and t.device != device:
            raise ValueError(f"tensors on {device} and {t.device}")


def _drop(d):
    return B.TngDrop(int(d.seed) & 0xFFFFFFFFFFFFFFFF, int(d.iter) & 0xFFFFFFFF, int(d.site), float(d.p), int(bool(d.relu)))


def _stream(device):
    return ctypes.c_void_p(torch.cuda.current_stream(device).cuda_stream)


def _scratch(nbytes, device):
    # (the library sizes what it refuses as 0, and says so when it is called)
    return torch.empty(nbytes, dtype=torch.uint8, device=device)


def _codes(shape, device):
    """int8 codes whose rows begin 16 bytes apart, which the products' fast kernels ask for."""
    cols = shape[-1]
    held = torch.empty((*shape[:-1], -(-cols // 16) * 16), dtype=torch.int8, device=device)
    return held[..., :cols]


def _out(out, shape, dtype, device, name):
    if out is None:
        return torch.empty(shape, dtype=dtype, device=device)
    if tuple(out.shape) != tuple(shape) or out.dtype != dtype or out.device != device:
        raise ValueError(f"{name}: expected {tuple(shape)} {dtype} on {device}")
    return out


def dropout(x, drop, residual=None, out=None):
    """keep f(x) / (1 - p), plus the residual if there is one."""
    mx = _matrix(x, _TYPES, "x")
    out = _out(out, x.shape, x.dtype, x.device, "out")
    _same_device(x.device, residual)
    mr = None if residual is None else _matrix(residual, _TYPES, "residual")
    with torch.cuda.device(x.device):
        B._check(B.lib().tng_dropout(_stream(x.device), _drop(drop), mx, mr, _matrix(out, _TYPES, "out")), "tng_dropout")
    return out


def dropout_grad(dy, drop, x=None, out=None):
    """The gradient of dropout's x from that of its result; x is needed if there is a relu."""
    md = _matrix(dy, _TYPES, "dy")
    out = _out(out, dy.shape, dy.dtype, dy.device, "out")
    _same_device(dy.device, x)
    mx = None if x is None else _matrix(x, _TYPES, "x")
    with torch.cuda.device(dy.device):
        B._check(B.lib().tng_dropout_grad(_stream(dy.device), _drop(drop), mx, md, _matrix(out, _TYPES, "out")), "tng_dropout_grad")
    return out


def quantize_rows(x, drop=None, turned=False):
    """(codes, scales) of x's rows, or of what drop makes of them; turned: (codes, scales, turned codes)."""
    mx = _matrix(x, _TYPES, "x")
    q = _codes(x.shape, x.device)
    scale = torch.empty(x.shape[:-1], dtype=torch.float32, device=x.device)
    qt = _codes((*x.shape[:-2], x.shape[-1], x.shape[-2]), x.device) if turned else None
    with torch.cuda.device(x.device):
        B._check(B.lib().tng_quantize_rows(_stream(x.device), None if drop is None else _drop(drop), mx, _matrix(q, _I8, "q"),
                                           scale.data_ptr(), None if qt is None else _matrix(qt, _I8, "qt")), "tng_quantize_rows")
    return (q, scale, qt) if turned else (q, scale)


def weight(w, turned=True):
    """The codes of a layer's weights [channels, depth], laid out once for every use until they change."""
    return Weight(*quantize_rows(w, turned=turned))


def quantize_grad(dy, col_scale=None, row_scale=None, *, seed, iter, site, sums=True):
    """(q, q_scale, qt, qt_scale, col_sum): the codes of dy col_scale by rows and of dy row_scale by columns, and dy's column sums."""
    m = _matrix(dy, _TYPES, "dy")
    dev, lead = dy.device, dy.shape[:-2]
    rows, cols = dy.shape[-2:]
    q, qt = _codes(dy.shape, dev), _codes((*lead, cols, rows), dev)
    q_scale = torch.empty((*lead, rows), dtype=torch.float32, device=dev)
    qt_scale = torch.empty((*lead, cols), dtype=torch.float32, device=dev)
    col_sum = torch.empty((*lead, cols), dtype=torch.float32, device=dev) if sums else None
    scratch = _scratch(B.lib().tng_quantize_grad_bytes(m), dev)
    with torch.cuda.device(dev):
        B._check(B.lib().tng_quantize_grad(
            _stream(dev), _drop(Drop(seed, iter, site)), m, _vector(col_scale, cols, "col_scale", dev),
            _vector(row_scale, m.workers * rows, "row_scale", dev), _matrix(q, _I8, "q"), q_scale.data_ptr(), _matrix(qt, _I8, "qt"),
            qt_scale.data_ptr(), col_sum.data_ptr() if sums else None, scratch.data_ptr(), scratch.numel()), "tng_quantize_grad")
    return q, q_scale, qt, qt_scale, col_sum


def matmul_i8(a, b, a_scale=None, b_scale=None, bias=None, dtype=torch.float32, out=None, drop=None, x=None):
    """a_scale b_scale (a b^T) + bias: codes a [rows, depth] or [M, rows, depth], b [channels, depth] or one for each worker.
    drop, x: the result is a gradient that goes on through that dropout (and its relu, of x)."""
    ma, mb = _matrix(a, _I8, "a"), _matrix(b, _I8, "b")
    dev = a.device
    _same_device(dev, b, x)
    out = _out(out, (*a.shape[:-1], b.shape[-2]), dtype, dev, "out")
    my = _matrix(out, _TYPES, "out")
    mx = None if x is None else _matrix(x, _TYPES, "x")
    L = B.lib()
    scratch = _scratch(L.tng_matmul_i8_bytes(ma, mb, my), dev)
    with torch.cuda.device(dev):
        B._check(L.tng_matmul_i8(
            _stream(dev), ma, _vector(a_scale, ma.workers * ma.rows, "a_scale", dev), mb,
            _vector(b_scale, mb.workers * mb.rows, "b_scale", dev), _vector(bias, mb.rows, "bias", dev),
            None if drop is None else _drop(drop), mx, my, scratch.data_ptr(), scratch.numel()), "tng_matmul_i8")
    return out


def linear(x, weight, bias=None, drop=None, keep=False):
    """The layer's result of x's type: the rows of x (of what drop makes of them) are coded and multiplied by the weights' codes.
    keep: also what linear_grad needs of this pass."""
    if keep:
        q, scale, qt = quantize_rows(x, drop, turned=True)
    else:
        q, scale = quantize_rows(x, drop)
    y = matmul_i8(q, weight.q, scale, weight.scale, bias, dtype=x.dtype)
    if not keep:
        return y
    return y, Saved(x if drop is not None and drop.relu else None, drop, scale, qt)


def linear_grad(dy, saved, weight, *, seed, iter, site, out=None):
    """(dx, dw, db) from the gradient of linear's result: dx of dy's type, dw [M, channels, depth] and db [M, channels] float32
    (without the M where x had none).  The gradient is coded to 8 bits by unbiased draws of (seed, iter, site), and the derivative
    is that of the product of the codes, which stand for x and the weights.  out: where dw is written, any pitch."""
    if weight.qt is None:
        raise ValueError("linear_grad needs the weights' turned codes")
    q, q_scale, qt, qt_scale, db = quantize_grad(dy, weight.scale, saved.scale, seed=seed, iter=iter, site=site)
    dx = matmul_i8(q, weight.qt, q_scale, dtype=dy.dtype, drop=saved.drop, x=saved.x)
    dw = matmul_i8(qt, saved.qt, qt_scale, out=out)
    return dx, dw, db
