"""8-bit operands with a scale for each block of 128, and the linear layer of them
(mag_quantize_fp8, mag_linear_fp8 in include/magneton.h).

Calls, buffers and streams as in the block's other operators: asynchronous on the
current stream of the tensors' device, on values (no gradient is recorded).  The
gradients of a layer are such products themselves:

    q, s, qt, st = quantize_fp8(x, transposed=True)             # rows, and columns
    w, ws, wt, wst = quantize_fp8(weight, 128, transposed=True)
    y = linear_fp8(q, s, w, ws)
    d, ds, dt, dst = quantize_fp8(dy, transposed=True)
    dx = linear_fp8(d, ds, wt, wst)          # dy weight
    dweight = linear_fp8(dt, dst, qt, st)    # dy^T x
"""
from __future__ import annotations

import torch

from . import MagnetonError, _lib
from . import _native as N
from ._block import (_NONE, _activation, _as_rows, _dtype, _launch, _matrix, _refuse, _size,
                     _vector, _workspace)

BLOCK = 128
_FORMATS = {torch.float8_e4m3fn: N.MAG_E4M3, torch.float8_e5m2: N.MAG_E5M2}


def _format(x, name):
    if not isinstance(x, torch.Tensor) or not x.is_cuda:
        raise MagnetonError(N.MAG_E_NULL, f"{name} must be a GPU tensor")
    try:
        return _FORMATS[x.dtype]
    except KeyError:
        raise MagnetonError(N.MAG_E_SIZE, f"{name} must be float8_e4m3fn or float8_e5m2, "
                                          f"got {x.dtype}") from None


def _blocks(n):
    return -(-n // BLOCK)


def _pitch(n):
    """bytes from a row of n to the next: whole lines, but for narrow rows"""
    return -(-n // 128) * 128 if n > 128 else -(-n // 16) * 16


def _new_rows(rows, cols, dtype, device):
    return torch.empty((rows, _pitch(cols)), dtype=dtype, device=device)[:, :cols]


def _new_scales(rows, cols, device):
    # (stored by columns: a product reads the scales of many rows and one block at once)
    return torch.empty((cols, rows), dtype=torch.float32, device=device).t()


def quantize_fp8(x, block_rows=1, *, dtype=torch.float8_e4m3fn, transposed=False, out=None):
    """x in 8 bits with a float32 scale for each block, q scale = x as nearly as q's
    type allows: scale = max(largest magnitude of the block / largest number of the
    type, 2^-126), q = x / scale rounded to nearest.

    x: [..., cols], float32, float16 or bfloat16, any strides.  block_rows: 1 for blocks
    of 1 x 128 (activations), 128 for 128 x 128 (weights).  dtype: float8_e4m3fn or
    float8_e5m2.  Returns (q, scale): q [rows, cols] in rows of whole 16 bytes (a
    view), scale [rows or ceil(rows / 128), ceil(cols / 128)], stored by columns;
    leading dimensions come as one.  transposed: (q, scale, qt, scale_t), with those of
    x's transpose.  out: the tensors to write.
    """
    lib = _lib()
    dt = _dtype(x, "x")
    try:
        fmt = _FORMATS[dtype]
    except (KeyError, TypeError):
        raise MagnetonError(N.MAG_E_SIZE, f"unknown 8-bit type {dtype!r}") from None
    x = _as_rows(x, "x")
    index = x.get_device()
    rows, cols = x.shape
    if out is None:
        tall = rows if block_rows == 1 else _blocks(rows)
        out = (_new_rows(rows, cols, dtype, x.device), _new_scales(tall, _blocks(cols), x.device))
        if transposed:
            wide = cols if block_rows == 1 else _blocks(cols)
            out += (_new_rows(cols, rows, dtype, x.device), _new_scales(wide, _blocks(rows), x.device))
    elif len(out) != (4 if transposed else 2):
        raise MagnetonError(N.MAG_E_SIZE, "out must be (q, scale), transposed (q, scale, qt, scale_t)")
    given = [_matrix(t, dtype if i % 2 == 0 else torch.float32, index, name)
             for i, (t, name) in enumerate(zip(out, ("q", "scale", "qt", "scale_t")))]
    given += [_NONE] * (4 - len(given))
    args = N.QUANTIZE_ARGS.pack(dt, fmt, int(block_rows), 0, *_matrix(x, x.dtype, index, "x"),
                                *given[0], *given[1], *given[2], *given[3])
    _launch(index, lib.mag_quantize_fp8, args)
    return out


def _linear_args(x, x_scale, weight, weight_scale, bias, residual, act, pre, out):
    fx, fw, dev = _format(x, "x"), _format(weight, "weight"), x.get_device()
    mw = _matrix(weight, weight.dtype, dev, "weight")
    if out is None:
        ty, dt = torch.bfloat16, N.MAG_BF16
    else:
        dt, ty = _dtype(out, "out"), out.dtype
    return N.LINEAR_FP8_ARGS.pack(
        dt, act, fx, fw, *_matrix(x, x.dtype, dev, "x"), *mw,
        *(_NONE if residual is None else _matrix(residual, ty, dev, "residual")),
        *(_NONE if pre is None else _matrix(pre, ty, dev, "pre")),
        *(_NONE if out is None else _matrix(out, ty, dev, "out")),
        *(_NONE if x_scale is None else _matrix(x_scale, torch.float32, dev, "x_scale")),
        *(_NONE if weight_scale is None else _matrix(weight_scale, torch.float32, dev, "weight_scale")),
        0 if bias is None else _vector(bias, ty, dev, mw[1], "bias"))


def linear_fp8_workspace_size(x, weight) -> int:
    return _size(_lib().mag_linear_fp8_workspace_size,
                 _linear_args(x, None, weight, None, None, None, 0, None, None))


def linear_fp8(x, x_scale, weight, weight_scale, bias=None, residual=None, *, activation=None,
               pre=None, out=None, dtype=torch.bfloat16, workspace=None):
    """act(x weight^T + bias) + residual of 8-bit operands in one pass over the product:
    linear() of what quantize_fp8 returns.

    x: [..., in], weight: [out, in], float8_e4m3fn or float8_e5m2, any strides (rows of
    whole 16 bytes are read where they lie).  x_scale: [rows, ceil(in / 128)];
    weight_scale: [ceil(out / 128), ceil(in / 128)], or one for each output's block, [out,
    ceil(in / 128)]; float32, rows up to 2^22 values apart.  bias: [out], residual: [..., out], of dtype
    (float16 or bfloat16; out's, where it is given).  activation, pre, out: as in linear();
    residual may be `out` itself.  Returns out, or (out, pre), which carry no gradient.
    """
    lib = _lib()
    act = _activation(activation)
    _format(x, "x")
    for t, name in ((x_scale, "x_scale"), (weight_scale, "weight_scale")):
        if not isinstance(t, torch.Tensor):
            _refuse(t, torch.float32, x.get_device(), name)
    if out is None or pre is True:
        if not isinstance(weight, torch.Tensor) or weight.dim() != 2:
            raise MagnetonError(N.MAG_E_SIZE, "weight must be [out, in]")
        shape = (*x.shape[:-1], weight.shape[0])
        if out is None:
            out = torch.empty(shape, dtype=dtype, device=x.device)
        if pre is True:
            pre = torch.empty(shape, dtype=out.dtype, device=x.device)
    args = _linear_args(x, x_scale, weight, weight_scale, bias, residual, act, pre, out)
    ws, p, n = _workspace(workspace, lib.mag_linear_fp8_workspace_size, args, x)
    _launch(x.get_device(), lib.mag_linear_fp8, args, p, n)
    return out if pre is None else (out, pre)
