"""The operators of a feed-forward block: linear layers with bias, activation
and residual in one pass, layer norms, their gradients, and the
orthogonalisation of a weight's update (mag_linear ... mag_orthogonalize in
include/magneton.h).

Every call is asynchronous on the current stream of its tensors' device.
Outputs and workspaces may be given (`out`, `workspace`: a program that calls
in a loop keeps them) and are allocated otherwise.

These are operators on values, as the rest of this package: autograd does not see
them.  Results of tensors that require a gradient carry none; linear_backward and
layer_norm_backward compute it.
"""
from __future__ import annotations

import ctypes

import torch

from . import MagnetonError, _check, _lib
from . import _native as N

_DTYPES = {torch.float32: N.MAG_F32, torch.float16: N.MAG_F16, torch.bfloat16: N.MAG_BF16}
_ACTIVATIONS = {None: N.MAG_ACT_NONE, "none": N.MAG_ACT_NONE, "relu": N.MAG_ACT_RELU,
                "gelu": N.MAG_ACT_GELU, "gelu_tanh": N.MAG_ACT_GELU_TANH, "silu": N.MAG_ACT_SILU}
_NONE = (0, 0, 0, 0, 0)


def _dtype(x, name):
    if not isinstance(x, torch.Tensor) or not x.is_cuda:
        raise MagnetonError(N.MAG_E_NULL, f"{name} must be a GPU tensor")
    try:
        return _DTYPES[x.dtype]
    except KeyError:
        raise MagnetonError(N.MAG_E_SIZE, f"{name} must be float32, float16 or bfloat16, "
                                          f"got {x.dtype}") from None


def _as_rows(x, name):
    """x with its leading dimensions as one (a view; never a copy)"""
    if x.dim() == 2:
        return x
    if x.dim() == 0:
        raise MagnetonError(N.MAG_E_SIZE, f"{name} has no dimension")
    if x.dim() == 1:
        return x[None]
    rows = 1
    for n in x.shape[:-1]:
        rows *= n
    try:
        return x.view(rows, x.shape[-1])
    except RuntimeError:
        raise MagnetonError(N.MAG_E_SIZE, f"{name}: the leading dimensions of strides "
                                          f"{x.stride()} cannot be seen as one") from None


def _refuse(x, dtype, index, name):
    """why x is not what _matrix or _vector ask for"""
    if not isinstance(x, torch.Tensor) or x.get_device() != index:
        raise MagnetonError(N.MAG_E_NULL, f"{name} must be a tensor on GPU {index}")
    raise MagnetonError(N.MAG_E_SIZE, f"{name} must be {dtype}, got {x.dtype}")


# (a decode step calls these some ten times: few attribute reads, one check)
def _matrix(x, dtype, index, name):
    """The five fields of a mag_matrix; x: a tensor of that type and device."""
    if not isinstance(x, torch.Tensor) or x.dtype is not dtype or x.get_device() != index:
        _refuse(x, dtype, index, name)
    if x.dim() != 2:
        x = _as_rows(x, name)
    return (x.data_ptr(), *x.shape, *x.stride())


def _vector(x, dtype, index, width, name):
    if not isinstance(x, torch.Tensor) or x.dtype is not dtype or x.get_device() != index:
        _refuse(x, dtype, index, name)
    if x.shape != (width,) or not x.is_contiguous():
        raise MagnetonError(N.MAG_E_SIZE, f"{name} must be {width} contiguous values")
    return x.data_ptr()


def _activation(kind):
    try:
        return _ACTIVATIONS[kind]
    except (KeyError, TypeError):
        raise MagnetonError(N.MAG_E_SIZE, f"unknown activation {kind!r}") from None


def _size(call, args) -> int:
    b = ctypes.c_size_t(0)
    _check(call(args, ctypes.byref(b)))
    return int(b.value)


def _workspace(workspace, size, args, like):
    """(tensor, pointer, bytes) of the workspace given, or of one allocated for the
    call (its memory is reused in stream order)."""
    if workspace is None:
        bytes_ = _size(size, args)
        if not bytes_:
            return None, 0, 0
        workspace = torch.empty(bytes_, dtype=torch.uint8, device=like.device)
    elif (not isinstance(workspace, torch.Tensor) or workspace.get_device() != like.get_device()
          or not workspace.is_contiguous()):
        raise MagnetonError(N.MAG_E_WORKSPACE, f"workspace must be contiguous on {like.device}")
    return workspace, workspace.data_ptr(), workspace.numel() * workspace.element_size()


# the handle of a device's current stream without a stream object around it
_raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None) or (
    lambda index: torch.cuda.current_stream(index).cuda_stream)


def _launch(index, call, *args):
    """call(*args, stream) with the tensors' device current"""
    if index == torch.cuda.current_device():
        rc = call(*args, _raw_stream(index))
    else:
        with torch.cuda.device(index):
            rc = call(*args, _raw_stream(index))
    if rc:
        _check(rc)


def _linear_args(x, weight, bias, residual, act, pre, out):
    dt, ty, dev = _dtype(x, "x"), x.dtype, x.get_device()
    mw = _matrix(weight, ty, dev, "weight")
    return N.LINEAR_ARGS.pack(
        dt, act, *_matrix(x, ty, dev, "x"), *mw,
        *(_NONE if residual is None else _matrix(residual, ty, dev, "residual")),
        *(_NONE if pre is None else _matrix(pre, ty, dev, "pre")),
        *(_NONE if out is None else _matrix(out, ty, dev, "out")),
        0 if bias is None else _vector(bias, ty, dev, mw[1], "bias"))


def linear_workspace_size(x, weight) -> int:
    return _size(_lib().mag_linear_workspace_size,
                 _linear_args(x, weight, None, None, 0, None, None))


def linear(x, weight, bias=None, residual=None, *, activation=None, pre=None, out=None,
           workspace=None):
    """act(x weight^T + bias) + residual in one pass over the product.

    x: [..., in], weight: [out, in], any strides (a transposed view for a weight
    stored input by output), bias: [out], residual: [..., out]; one type, float32,
    float16 or bfloat16.  activation: None, "relu", "gelu", "gelu_tanh", "silu".
    pre: True, or a tensor, for x weight^T + bias as well (what linear_backward
    reads).  residual may be `out` itself.  Returns out, or (out, pre), which carry
    no gradient: call linear_backward for it.
    """
    lib = _lib()
    act = _activation(activation)
    _dtype(x, "x")
    if out is None or pre is True:
        if not isinstance(weight, torch.Tensor) or weight.dim() != 2:
            raise MagnetonError(N.MAG_E_SIZE, "weight must be [out, in]")
        shape = (*x.shape[:-1], weight.shape[0])
        if out is None:
            out = torch.empty(shape, dtype=x.dtype, device=x.device)
        if pre is True:
            pre = torch.empty(shape, dtype=x.dtype, device=x.device)
    args = _linear_args(x, weight, bias, residual, act, pre, out)
    ws, p, n = _workspace(workspace, lib.mag_linear_workspace_size, args, x)
    _launch(x.get_device(), lib.mag_linear, args, p, n)
    return out if pre is None else (out, pre)


def _linear_backward_args(x, weight, dy, pre, act, dx, dweight, dbias):
    dt, ty, dev = _dtype(x, "x"), x.dtype, x.get_device()
    mw = _matrix(weight, ty, dev, "weight")
    return N.LINEAR_BACKWARD_ARGS.pack(
        dt, act, *_matrix(x, ty, dev, "x"), *mw,
        *(_NONE if pre is None else _matrix(pre, ty, dev, "pre")),
        *(_NONE if dy is None else _matrix(dy, ty, dev, "dy")),
        *(_NONE if dx is None else _matrix(dx, ty, dev, "dx")),
        *(_NONE if dweight is None else _matrix(dweight, ty, dev, "dweight")),
        0 if dbias is None else _vector(dbias, ty, dev, mw[1], "dbias"))


def linear_backward_workspace_size(x, weight, dy=None) -> int:
    """Bytes for these tensors; without dy, for a dy of any strides."""
    return _size(_lib().mag_linear_backward_workspace_size,
                 _linear_backward_args(x, weight, dy, None, 0, None, None, None))


def linear_backward(x, weight, dy, pre=None, *, activation=None, bias=True,
                    need=(True, True), out=None, workspace=None):
    """Gradients of linear(): (dx, dweight, dbias), from its inputs, the gradient
    dy of its output and, with an activation, its `pre`.  need: whether dx and
    dweight are wanted; bias: whether dbias is (None is returned for the rest).
    The residual's gradient is dy.  out: three tensors to write (or None each)."""
    lib = _lib()
    act = _activation(activation)
    _dtype(x, "x")
    if out is None:
        if not isinstance(weight, torch.Tensor) or weight.dim() != 2:
            raise MagnetonError(N.MAG_E_SIZE, "weight must be [out, in]")
        new = dict(dtype=x.dtype, device=x.device)
        out = (torch.empty(x.shape, **new) if need[0] else None,
               torch.empty(weight.shape, **new) if need[1] else None,
               torch.empty(weight.shape[0], **new) if bias else None)
    dx, dweight, dbias = out
    args = _linear_backward_args(x, weight, dy, pre, act, dx, dweight, dbias)
    ws, p, n = _workspace(workspace, lib.mag_linear_backward_workspace_size, args, x)
    _launch(x.get_device(), lib.mag_linear_backward, args, p, n)
    return dx, dweight, dbias


def _norm_args(x, weight, bias, y, dy, dx, mean, rstd, dweight, dbias, eps):
    dt, ty, dev = _dtype(x, "x"), x.dtype, x.get_device()
    mx = _matrix(x, ty, dev, "x")
    _, rows, width, _, _ = mx
    wt, wdt = ty, dt
    for some in (weight, bias, dweight, dbias):
        if some is not None:
            wdt, wt = _dtype(some, "weight"), some.dtype
            break
    f32 = torch.float32
    return N.NORM_ARGS.pack(
        dt, wdt, *mx, *(_NONE if y is None else _matrix(y, ty, dev, "out")),
        *(_NONE if dy is None else _matrix(dy, ty, dev, "dy")),
        *(_NONE if dx is None else _matrix(dx, ty, dev, "dx")),
        0 if weight is None else _vector(weight, wt, dev, width, "weight"),
        0 if bias is None else _vector(bias, wt, dev, width, "bias"),
        0 if mean is None else _vector(mean, f32, dev, rows, "mean"),
        0 if rstd is None else _vector(rstd, f32, dev, rows, "rstd"),
        0 if dweight is None else _vector(dweight, wt, dev, width, "dweight"),
        0 if dbias is None else _vector(dbias, wt, dev, width, "dbias"), eps)


def layer_norm(x, weight=None, bias=None, eps=1e-5, *, statistics=None, out=None):
    """(x - mean) rstd weight + bias over the last dimension, rstd = 1 /
    sqrt(variance + eps).  weight and bias: [width], of x's type or float32, or
    None.  statistics: True, or two float32 tensors of one value per row, for
    the mean and rstd too (what layer_norm_backward reads).  out may be x itself.
    Returns out, or (out, mean, rstd), which carry no gradient: call
    layer_norm_backward for it."""
    lib = _lib()
    if out is None:
        _dtype(x, "x")
        out = torch.empty(x.shape, dtype=x.dtype, device=x.device)
    mean = rstd = None
    if statistics is True:
        rows = _as_rows(x, "x").shape[0]
        mean, rstd = (torch.empty(rows, device=x.device) for _ in range(2))
    elif statistics is not None:
        mean, rstd = statistics
    args = _norm_args(x, weight, bias, out, None, None, mean, rstd, None, None, eps)
    _launch(x.get_device(), lib.mag_layer_norm, args)
    return out if statistics is None else (out, mean, rstd)


def layer_norm_backward_workspace_size(x) -> int:
    return _size(_lib().mag_layer_norm_backward_workspace_size,
                 _norm_args(x, None, None, None, None, None, None, None, None, None, 0.0))


def layer_norm_backward(x, dy, mean, rstd, weight=None, *, need=(True, True, True), out=None,
                        workspace=None):
    """Gradients of layer_norm(): (dx, dweight, dbias), from its input, the
    gradient dy of its output and the statistics it returned.  need: which are
    wanted (None for the rest).  out: three tensors to write (or None each); dx
    may be x or dy itself.  dweight and dbias have weight's type (float32 without
    a weight)."""
    lib = _lib()
    _dtype(x, "x")
    if weight is not None:
        _dtype(weight, "weight")
    if out is None:
        wt = torch.float32 if weight is None else weight.dtype
        out = (torch.empty(x.shape, dtype=x.dtype, device=x.device) if need[0] else None,
               torch.empty(x.shape[-1], dtype=wt, device=x.device) if need[1] else None,
               torch.empty(x.shape[-1], dtype=wt, device=x.device) if need[2] else None)
    dx, dweight, dbias = out
    args = _norm_args(x, weight, None, None, dy, dx, mean, rstd, dweight, dbias, 0.0)
    ws, p, n = _workspace(workspace, lib.mag_layer_norm_backward_workspace_size, args, x)
    _launch(x.get_device(), lib.mag_layer_norm_backward, args, p, n)
    return dx, dweight, dbias


def _orthogonalize_args(g, steps, coefficients, eps, out):
    dt = _dtype(g, "g")
    if out is None:
        out = g
    elif not isinstance(out, torch.Tensor) or out.get_device() != g.get_device():
        raise MagnetonError(N.MAG_E_NULL, f"out must be a tensor on {g.device}")
    if g.dim() not in (2, 3) or out.shape != g.shape:
        raise MagnetonError(N.MAG_E_SIZE, "g and out must be [rows, cols] or [batch, rows, cols]")
    if out.dtype != g.dtype:
        raise MagnetonError(N.MAG_E_SIZE, f"out must be {g.dtype}, got {out.dtype}")
    batch = g.shape[0] if g.dim() == 3 else 1
    a, b, c = coefficients
    return N.ORTHOGONALIZE_ARGS.pack(
        dt, int(steps), batch, g.data_ptr(), *g.shape[-2:], *g.stride()[-2:], out.data_ptr(),
        *out.shape[-2:], *out.stride()[-2:], g.stride(0) if g.dim() == 3 else 0,
        out.stride(0) if g.dim() == 3 else 0, float(a), float(b), float(c), float(eps))


def orthogonalize_workspace_size(g) -> int:
    return _size(_lib().mag_orthogonalize_workspace_size,
                 _orthogonalize_args(g, 1, (1.0, 0.0, 0.0), 0.0, None))


def orthogonalize(g, steps=5, coefficients=(3.4445, -4.7750, 2.0315), eps=1e-7, *, out=None,
                  workspace=None):
    """An update with its singular values driven towards one (Newton-Schulz):
    X = g / (|g| + eps), then `steps` times X <- a X + (b A + c A A) X with A = X
    X^T (on the transpose where g is taller than wide).  g: [rows, cols], or
    [batch, rows, cols] for several on their own.  out may be g itself.  The result
    carries no gradient."""
    lib = _lib()
    _dtype(g, "g")
    if out is None:
        out = torch.empty(g.shape, dtype=g.dtype, device=g.device)
    args = _orthogonalize_args(g, steps, coefficients, eps, out)
    ws, p, n = _workspace(workspace, lib.mag_orthogonalize_workspace_size, args, g)
    _launch(g.get_device(), lib.mag_orthogonalize, args, p, n)
    return out
