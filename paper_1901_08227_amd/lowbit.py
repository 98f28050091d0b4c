"""Linear layers of libtng's simulated workers in 8-bit codes, and dropout whose mask is never stored (the layer calls of
include/tng.h on torch tensors).

Tensors are [rows, cols] for one worker or [M, rows, cols] for M of them, float32, bfloat16 or float16, on the GPU, with contiguous
rows.  The strides of rows and workers are free as long as a worker's matrix ends before the next one begins (inputs may also have
strides of 0; workers whose rows alternate are refused).  Everything runs in the library's kernels on the current stream of the
tensors' device; results and scratch come from torch's allocator.  A training step of a layer is

    y, saved = linear(x, weight, bias, drop, keep=True)
    dx, dw, db = linear_grad(dy, saved, weight, seed=..., iter=..., site=...)

with dw and db of every worker, as the coder of the gradients takes them (out= puts dw where g[M][d] has it).

Nothing here is recorded by autograd: what the calls make never requires a gradient, also where an argument does, and the backward
pass is the calls above.
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
    which the backward pass reads.  With a leading M each worker has weights of its own: a layer then answers, but linear_grad
    takes one set of weights for all workers only."""
    q: torch.Tensor
    scale: torch.Tensor
    qt: Optional[torch.Tensor] = None


class Saved(NamedTuple):
    """What the backward pass of a layer reads again of its forward pass.  x is the caller's tensor, not a copy: what is written to it
    before linear_grad changes which elements the relu lets through."""
    x: Optional[torch.Tensor]  # only where a relu's gradient needs it
    drop: Optional[Drop]
    scale: torch.Tensor        # of the tokens' codes, [M, rows]
    qt: torch.Tensor           # the tokens' codes turned, [M, depth, rows]


_I8 = {torch.int8: B.TYPE_I8}
# The arguments of the layer calls behind the stream, a letter each (see csrc/tng_call.cpp), what they are called here, and the letters of a
# call that makes its result.
_CALLS = {
    "tng_dropout": ("dmmm", ("drop", "x", "residual", "out"), "dmmo"),
    "tng_dropout_grad": ("dmmm", ("drop", "x", "dy", "out"), None),
    "tng_quantize_rows": ("dmiri", ("drop", "x", "q", "scale", "qt"), None),
    "tng_quantize_grad": ("dmcririrrw", ("key", "dy", "col_scale", "row_scale", "q", "q_scale", "qt", "qt_scale", "col_sum"), None),
    "tng_matmul_i8": ("irirndmmW", ("a", "a_scale", "b", "b_scale", "bias", "drop", "x", "out"), None),
    "tng_linear_i8": ("dmirnmW", ("drop", "x", "codes", "scale", "bias", "out"), "dmirnpW"),
}


def _u32(n):
    """n as 32 bits; what they do not hold as the largest number, which the library refuses for every field that this is used for."""
    return n if 0 <= n < 1 << 32 else 0xFFFFFFFF


def _matrix(t, dtypes, name):
    """The tng_matrix of a tensor."""
    if not isinstance(t, torch.Tensor) or not t.is_cuda:
        raise TypeError(f"{name}: expected a CUDA tensor")
    kind = dtypes.get(t.dtype)
    if kind is None:
        raise TypeError(f"{name}: {t.dtype} is not one of {', '.join(map(str, dtypes))}")
    shape, stride = t.shape, t.stride()
    if len(shape) == 2:
        workers, pitch = 1, 0
    elif len(shape) == 3:
        workers, pitch = _u32(shape[0]), stride[0]
    else:
        raise ValueError(f"{name}: expected [rows, cols] or [M, rows, cols], got {tuple(shape)}")
    if stride[-1] != 1 and shape[-1] > 1:
        raise TypeError(f"{name}: rows have to be contiguous")
    return B.TngMatrix(t.data_ptr(), kind, workers, shape[-2], shape[-1], stride[-2], pitch)


def _vector(t, n, name):
    """Address of a contiguous float32 tensor of n elements."""
    if not isinstance(t, torch.Tensor) or not t.is_cuda or t.dtype != torch.float32 or not t.is_contiguous():
        raise TypeError(f"{name}: expected contiguous float32 on the GPU")
    if t.numel() != n:
        raise ValueError(f"{name}: needs {n} elements, has {t.numel()}")
    return t.data_ptr()


def _drop(d):
    return B.TngDrop(int(d[0]) & 0xFFFFFFFFFFFFFFFF, int(d[1]) & 0xFFFFFFFF, _u32(int(d[2])), float(d[3]), int(bool(d[4])))


def _through_ctypes(name, kinds, names, device, stream, args):
    """The call with arguments that the native function does not take as plain: converts them, or says what is wrong."""
    L, values, matrices = B.lib(), [], []
    for kind, what, arg in zip(kinds, names, args):
        if isinstance(arg, torch.Tensor) and arg.is_cuda and arg.device != device:
            raise ValueError(f"{what}: on {arg.device}, the others on {device}")
        if arg is None:
            values.append(None)
        elif kind == "d":
            values.append(_drop(arg))
        elif kind in "mi":
            values.append(_matrix(arg, _TYPES if kind == "m" else _I8, what))
            matrices.append(values[-1])
        else:
            m = matrices[-1]
            values.append(_vector(arg, {"r": m.workers * m.rows, "n": m.rows, "c": m.cols}[kind], what))
    if kinds[-1] in "wW":  # (the library sizes what it refuses as 0, and says so when it is called)
        sized = matrices[:1] if kinds[-1] == "w" else [*matrices[:2], matrices[-1]]
        scratch = torch.empty(getattr(L, name + "_bytes")(*sized), dtype=torch.uint8, device=device)
        values += [scratch.data_ptr(), scratch.numel()]
    return getattr(L, name)(ctypes.c_void_p(stream), *values)


def _stream(device):
    return torch._C._cuda_getCurrentRawStream(device.index)


def _plain(device):
    """Whether the whole layer may be tried by the native function: on the current GPU."""
    B.lib()
    return device.type == "cuda" and device.index == torch.cuda.current_device()


_entries = None


def _layer_entries():
    global _entries
    if _entries is None:
        _entries = tuple(B._address[n] for n in ("tng_quantize_rows", "tng_quantize_grad", "tng_quantize_grad_bytes", "tng_matmul_i8",
                                                 "tng_matmul_i8_bytes"))
    return _entries


def _run(name, device, *args, made=None):
    """A layer call on the current stream of the device, by the native function where its arguments are plain.  made: the shape of the
    result, which is like the first matrix but for its columns, if there is none among the arguments; the native function makes it."""
    if device.type != "cuda":
        raise TypeError(f"{name}: expected CUDA tensors")
    if device.index != torch.cuda.current_device():
        with torch.cuda.device(device):
            return _run(name, device, *args, made=made)
    B.lib()
    kinds, names, makes = _CALLS[name]
    stream = _stream(device)
    status = B._layer(B._address[name], B._address.get(name + "_bytes", 0), stream, makes if made else kinds, *args)
    if status is None:
        if made:
            args = (*args, torch.empty(made, dtype=args[1].dtype, device=device))
        status = _through_ctypes(name, kinds, names, device, stream, args)
    elif not isinstance(status, int):
        return status
    B._check(status, name)
    return args[-1]


def _codes(shape, device):
    """int8 codes whose rows begin 16 bytes apart, which the products' fast kernels ask for."""
    cols = shape[-1]
    if cols % 16 == 0:
        return torch.empty(shape, dtype=torch.int8, device=device)
    return torch.empty((*shape[:-1], -(-cols // 16) * 16), dtype=torch.int8, device=device)[..., :cols]


def _floats(shape, device):
    return torch.empty(shape, dtype=torch.float32, device=device)


def _out(out, shape, dtype, device):
    if out is None:
        return torch.empty(shape, dtype=dtype, device=device)
    if tuple(out.shape) != tuple(shape) or out.dtype != dtype or out.device != device:
        raise ValueError(f"out: expected {tuple(shape)} {dtype} on {device}")
    return out


def _dims(t, name):
    if t.dim() not in (2, 3):
        raise ValueError(f"{name}: expected [rows, cols] or [M, rows, cols], got {tuple(t.shape)}")
    return t.shape


def dropout(x, drop, residual=None, out=None):
    """keep f(x) / (1 - p), plus the residual if there is one."""
    if out is None:
        return _run("tng_dropout", x.device, drop, x, residual, made=x.shape)
    return _run("tng_dropout", x.device, drop, x, residual, _out(out, x.shape, x.dtype, x.device))


def dropout_grad(dy, drop, x=None, out=None):
    """The gradient of dropout's x from that of its result; x is needed if there is a relu."""
    return _run("tng_dropout_grad", dy.device, drop, x, dy, _out(out, dy.shape, dy.dtype, dy.device))


def quantize_rows(x, drop=None, turned=False):
    """(codes, scales) of x's rows, or of what drop makes of them; turned: (codes, scales, turned codes)."""
    shape, device = _dims(x, "x"), x.device
    q, scale = _codes(shape, device), _floats(shape[:-1], device)
    qt = _codes((*shape[:-2], shape[-1], shape[-2]), device) if turned else None
    _run("tng_quantize_rows", device, drop, x, q, scale, qt)
    return (q, scale, qt) if turned else (q, scale)


def weight(w, turned=True):
    """The codes of a layer's weights [channels, depth], laid out once for every use until they change."""
    return Weight(*quantize_rows(w, turned=turned))


def quantize_grad(dy, col_scale=None, row_scale=None, *, seed, iter, site, sums=True):
    """(q, q_scale, qt, qt_scale, col_sum): the codes of dy col_scale by rows and of dy row_scale by columns, and dy's column sums."""
    (*lead, rows, cols), device = _dims(dy, "dy"), dy.device
    q, qt = _codes((*lead, rows, cols), device), _codes((*lead, cols, rows), device)
    q_scale, qt_scale = _floats((*lead, rows), device), _floats((*lead, cols), device)
    col_sum = _floats((*lead, cols), device) if sums else None
    _run("tng_quantize_grad", device, Drop(seed, iter, site), dy, col_scale, row_scale, q, q_scale, qt, qt_scale, col_sum)
    return q, q_scale, qt, qt_scale, col_sum


def matmul_i8(a, b, a_scale=None, b_scale=None, bias=None, dtype=torch.float32, out=None, drop=None, x=None):
    """a_scale b_scale (a b^T) + bias: codes a [rows, depth] or [M, rows, depth], b [channels, depth] or one for each worker.
    drop, x: the result is a gradient that goes on through that dropout (and its relu, of x)."""
    out = _out(out, (*_dims(a, "a")[:-1], _dims(b, "b")[-2]), dtype, a.device)
    return _run("tng_matmul_i8", a.device, a, a_scale, b, b_scale, bias, drop, x, out)


def linear(x, weight, bias=None, drop=None, keep=False):
    """The layer's result of x's type: the rows of x (of what drop makes of them) are coded and multiplied by the weights' codes.
    keep: also what linear_grad needs of this pass."""
    if not keep:
        made = (*_dims(x, "x")[:-1], _dims(weight.q, "codes")[-2])
        return _run("tng_linear_i8", x.device, drop, x, weight.q, weight.scale, bias, made=made)
    kept_x = x if drop is not None and drop.relu else None
    if _plain(x.device):
        got = B._linear(_layer_entries(), _stream(x.device), x, drop, weight.q, weight.scale, bias)
        if isinstance(got, int):
            B._check(got, "linear")
        if got is not None:
            return got[0], Saved(kept_x, drop, got[1], got[2])
    # (what is not plain: the calls one by one, which take it or say what is wrong)
    q, scale, qt = quantize_rows(x, drop, turned=True)
    return matmul_i8(q, weight.q, scale, weight.scale, bias, dtype=x.dtype), Saved(kept_x, drop, scale, qt)


def linear_grad(dy, saved, weight, *, seed, iter, site, out=None):
    """(dx, dw, db) from the gradient of linear's result: dx of dy's type, dw [M, channels, depth] and db [M, channels] float32
    (without the M where x had none).  The gradient is coded to 8 bits by unbiased draws of (seed, iter, site), and the derivative
    is that of the product of the codes, which stand for x and the weights.  out: where dw is written, any pitch."""
    if weight.qt is None:
        raise ValueError("linear_grad needs the weights' turned codes")
    if _plain(dy.device):
        got = B._linear_grad(_layer_entries(), _stream(dy.device), dy, saved.scale, saved.qt, weight.scale, weight.qt, saved.drop, saved.x,
                             (seed, iter, site, 0.0, False), out)
        if isinstance(got, int):
            B._check(got, "linear_grad")
        if got is not None:
            return got
    q, q_scale, qt, qt_scale, db = quantize_grad(dy, weight.scale, saved.scale, seed=seed, iter=iter, site=site)
    dx = matmul_i8(q, weight.qt, q_scale, dtype=dy.dtype, drop=saved.drop, x=saved.x)
    dw = matmul_i8(qt, saved.qt, qt_scale, out=out)
    return dx, dw, db
