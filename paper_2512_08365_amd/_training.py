"""What a training step adds around a block's layers: its norms fused with gate,
residual scale and addition, their gradients, and gradients clipped by their common
norm (mag_residual_norm ... mag_clip_gradients in include/magneton.h).

Calls, buffers and streams as in the block's other operators: asynchronous on the
current stream of the tensors' device, on values (no gradient is recorded).
"""
from __future__ import annotations

import math

import torch

from . import MagnetonError, _lib
from . import _native as N
from ._block import (_DTYPES, _NONE, _as_rows, _dtype, _launch, _matrix, _size, _vector, _workspace)

_KINDS = {"layer": N.MAG_NORM_LAYER, "rms": N.MAG_NORM_RMS}


def _kind(kind):
    try:
        return _KINDS[kind]
    except (KeyError, TypeError):
        raise MagnetonError(N.MAG_E_SIZE, f"unknown kind of norm {kind!r}") from None


def _first_dtype(tensors, otherwise):
    """the type that a call's weights share: the first one's"""
    for name, x in tensors:
        if x is not None:
            return _dtype(x, name), x.dtype
    return otherwise


def _optional(x, dtype, index, name):
    return _NONE if x is None else _matrix(x, dtype, index, name)


def _vectors(tensors, dtype, index, width):
    return [0 if x is None else _vector(x, dtype, index, width, name) for name, x in tensors]


_NO_STATISTICS = (0, 0, 0, 0)


def _statistics(stats, index, rows):
    if stats is None:
        return _NO_STATISTICS
    if len(stats) != 4:
        raise MagnetonError(N.MAG_E_SIZE, "statistics must be (mean, rstd, post_mean, post_rstd)")
    mean, rstd, post_mean, post_rstd = stats
    ty = torch.float32
    return (0 if mean is None else _vector(mean, ty, index, rows, "mean"),
            0 if rstd is None else _vector(rstd, ty, index, rows, "rstd"),
            0 if post_mean is None else _vector(post_mean, ty, index, rows, "post_mean"),
            0 if post_rstd is None else _vector(post_rstd, ty, index, rows, "post_rstd"))


def residual_norm(residual, branch, weight=None, bias=None, *, kind="rms", gate=None, scale=1.0,
                  post=False, post_weight=None, post_bias=None, eps=1e-5, statistics=None,
                  out=None):
    """The norms around a block in one pass: a = branch (with `post` its norm times
    post_weight + post_bias), stream = residual + scale gate a, normed = the norm of
    stream times weight + bias.

    residual, branch: [..., width], one type, float32, float16 or bfloat16.  kind: "rms"
    (x / sqrt(mean square + eps)) or "layer" ((x - mean) / sqrt(variance + eps)).  gate:
    [width], or [groups, width] for rows that come as `groups` samples of one length (a
    gate for every row: [rows, width]), of branch's type or float32.  Weights and biases:
    [width], one type, branch's or float32, or None.  statistics: True, or four float32
    tensors (mean, rstd, post_mean, post_rstd; None where not wanted) of one value a row,
    for what residual_norm_backward reads.  out: (stream, normed) to write; stream may be
    residual itself, normed branch.  Returns (stream, normed), or (stream, normed,
    statistics), which carry no gradient.
    """
    lib = _lib()
    dt, k = _dtype(branch, "branch"), _kind(kind)
    ty, dev = branch.dtype, branch.get_device()
    mr = _matrix(residual, ty, dev, "residual")
    _, rows, width, _, _ = mr
    if out is None:
        out = tuple(torch.empty(branch.shape, dtype=ty, device=branch.device) for _ in range(2))
    elif len(out) != 2:
        raise MagnetonError(N.MAG_E_SIZE, "out must be (stream, normed)")
    if statistics is True:
        layer = k == N.MAG_NORM_LAYER
        statistics = tuple(torch.empty(rows, device=branch.device) if on else None
                           for on in (layer, True, post and layer, post))
    # (a decode step calls this at every layer: no loops over what is mostly None)
    if weight is not None:
        wdt, wt = _dtype(weight, "weight"), weight.dtype
    else:
        wdt, wt = _first_dtype((("bias", bias), ("post_weight", post_weight), ("post_bias", post_bias)),
                               (dt, ty))
    gdt, gt = (dt, ty) if gate is None else (_dtype(gate, "gate"), gate.dtype)
    args = N.RESIDUAL_NORM_ARGS.pack(
        dt, wdt, gdt, k, bool(post), 0, *mr, *_matrix(branch, ty, dev, "branch"),
        *_matrix(out[0], ty, dev, "stream"), *_matrix(out[1], ty, dev, "normed"),
        *(_NONE if gate is None else _matrix(gate, gt, dev, "gate")),
        0 if weight is None else _vector(weight, wt, dev, width, "weight"),
        0 if bias is None else _vector(bias, wt, dev, width, "bias"),
        0 if post_weight is None else _vector(post_weight, wt, dev, width, "post_weight"),
        0 if post_bias is None else _vector(post_bias, wt, dev, width, "post_bias"),
        *(_NO_STATISTICS if statistics is None else _statistics(statistics, dev, rows)),
        float(scale), float(eps))
    _launch(dev, lib.mag_residual_norm, args)
    return (*out,) if statistics is None else (*out, tuple(statistics))


def _backward_args(stream, branch, d_normed, d_stream, statistics, weight, post_weight, post_bias,
                   kind, gate, scale, post, grads):
    dt, ty, dev = _dtype(stream, "stream"), stream.dtype, stream.get_device()
    ms = _matrix(stream, ty, dev, "stream")
    _, rows, width, _, _ = ms
    d_residual, d_branch, d_gate, *d_vectors = grads
    named = (("weight", weight), ("post_weight", post_weight), ("post_bias", post_bias))
    d_named = tuple(zip(("dweight", "dbias", "dpost_weight", "dpost_bias"), d_vectors))
    wdt, wt = _first_dtype((*named, *d_named), (dt, ty))
    gdt, gt = _first_dtype((("gate", gate),), (dt, ty))
    return N.RESIDUAL_NORM_BACKWARD_ARGS.pack(
        dt, wdt, gdt, kind, bool(post), 0, *ms, *_optional(branch, ty, dev, "branch"),
        *_optional(d_normed, ty, dev, "d_normed"), *_optional(d_stream, ty, dev, "d_stream"),
        *_optional(d_residual, ty, dev, "d_residual"), *_optional(d_branch, ty, dev, "d_branch"),
        *_optional(gate, gt, dev, "gate"), *_optional(d_gate, gt, dev, "d_gate"),
        *_vectors(named, wt, dev, width), *_statistics(statistics, dev, rows),
        *_vectors(d_named, wt, dev, width), float(scale))


def residual_norm_backward_workspace_size(stream, gate=None) -> int:
    return _size(_lib().mag_residual_norm_backward_workspace_size,
                 _backward_args(stream, None, None, None, None, None, None, None, 0, gate, 1.0, False,
                                (None,) * 7))


def residual_norm_backward(stream, branch, d_normed, d_stream, statistics, weight=None, bias=None,
                           *, kind="rms", gate=None, scale=1.0, post=False, post_weight=None,
                           post_bias=None, need=(True, True, True), out=None, workspace=None):
    """Gradients of residual_norm(): (d_residual, d_branch, d_gate, dweight, dbias,
    dpost_weight, dpost_bias), from its stream, its branch, the gradients of normed and
    (or None) of stream, and the statistics it returned.

    None is returned for what there is none of: the gate, weights and biases that are
    None (of a bias only its presence counts).  need: whether d_residual, d_branch and
    the rest are wanted.  out: seven tensors to write (or None each); d_residual may be
    d_stream itself, d_branch d_normed or branch.
    """
    lib = _lib()
    k = _kind(kind)
    _dtype(stream, "stream")
    if out is None:
        def like(x, wanted):
            return torch.empty(x.shape, dtype=x.dtype, device=stream.device) if wanted and x is not None else None

        out = (like(stream, need[0]), like(branch, need[1]),
               *(like(x, need[2]) for x in (gate, weight, bias, post_weight, post_bias)))
    elif len(out) != 7:
        raise MagnetonError(N.MAG_E_SIZE, "out must be seven tensors, or None each")
    args = _backward_args(stream, branch, d_normed, d_stream, statistics, weight, post_weight, post_bias,
                          k, gate, scale, post, out)
    ws, p, n = _workspace(workspace, lib.mag_residual_norm_backward_workspace_size, args, stream)
    _launch(stream.get_device(), lib.mag_residual_norm_backward, args, p, n)
    return (*out,)


# ----------------------------------------------------------------------- clipping

def _dense(x):
    """whether x's elements fill one run of memory, in whatever order"""
    at = 1
    for stride, size in sorted((s, n) for s, n in zip(x.stride(), x.shape) if n != 1):
        if stride != at:
            return False
        at *= size
    return True


def _place(x, y, name):
    """(cols, x's row stride, y's row stride) of tensors that are read and written"""
    if (x.is_contiguous() and y.is_contiguous()) or (x.stride() == y.stride() and _dense(x)):
        return 0, 0, 0
    rows = [_as_rows(t, name) for t in (x, y)]
    if any(r.shape[1] > 1 and r.stride(1) != 1 for r in rows):
        raise MagnetonError(N.MAG_E_SIZE, f"{name}: strides {x.stride()} and {y.stride()} are no rows of "
                                          "neighbours")
    return rows[0].shape[1], *(max(r.stride(0), r.shape[1]) if r.shape[0] == 1 else r.stride(0) for r in rows)


class TensorList:
    """Tensors of one GPU for gradient_norm and clip_gradients, described once: a program
    whose gradients stay where they are keeps it from step to step.  None among them
    is left out.  out: where clip_gradients writes them, in the tensors' types and shapes
    (None: the tensors themselves).  The list keeps the tensors."""

    def __init__(self, tensors, out=None):
        tensors = list(tensors)
        out = tensors if out is None else list(out)
        if len(out) != len(tensors):
            raise MagnetonError(N.MAG_E_SIZE, f"{len(tensors)} tensors and {len(out)} outputs")
        pairs = [(i, x, y) for i, (x, y) in enumerate(zip(tensors, out)) if x is not None]
        self.tensors, self.out = tuple(x for _, x, _ in pairs), tuple(y for _, _, y in pairs)
        self.index = None
        packed = bytearray(N.TENSOR_REF.size * len(pairs))
        for k, (i, x, y) in enumerate(pairs):
            name = f"tensor {i}"
            dt = _dtype(x, name)
            if self.index is None:
                self.index = x.get_device()
            for t in (x, y):
                if not isinstance(t, torch.Tensor) or t.get_device() != self.index:
                    raise MagnetonError(N.MAG_E_NULL, f"{name} must be on GPU {self.index}")
            if y.dtype is not x.dtype or y.shape != x.shape:
                raise MagnetonError(N.MAG_E_SIZE, f"{name}'s output must be {tuple(x.shape)} {x.dtype}")
            N.TENSOR_REF.pack_into(packed, k * N.TENSOR_REF.size, x.data_ptr(), y.data_ptr(), x.numel(),
                                   *_place(x, y, name), dt, 0)
        self._packed = bytes(packed)

    def __len__(self):
        return len(self.tensors)

    def _args(self, kind, max_norm, eps, norm):
        try:
            kind = {2: N.MAG_NORM_TWO, math.inf: N.MAG_NORM_INF}[kind]
        except (KeyError, TypeError):
            raise MagnetonError(N.MAG_E_SIZE, f"kind must be 2 or inf, got {kind!r}") from None
        return N.TENSORS_ARGS.pack(N.address(self._packed), len(self.tensors), kind, 0, float(max_norm),
                                   float(eps), 0 if norm is None else norm.data_ptr())


def _list(tensors, out=None):
    if isinstance(tensors, TensorList):
        if out is not None:
            raise MagnetonError(N.MAG_E_SIZE, "a TensorList has its own outputs")
        return tensors
    return TensorList(tensors, out)


def clip_gradients_workspace_size(tensors) -> int:
    tensors = _list(tensors)   # (kept: the arguments hold its address)
    return _size(_lib().mag_clip_gradients_workspace_size, tensors._args(2, 0.0, 0.0, None))


def _run(call, tensors, kind, max_norm, eps, norm, workspace):
    lib = _lib()
    if tensors.index is None:
        raise MagnetonError(N.MAG_E_SIZE, "the list has no tensor")
    if norm is None:
        norm = torch.empty((), dtype=torch.float32, device=tensors.tensors[0].device)
    elif (not isinstance(norm, torch.Tensor) or norm.dtype is not torch.float32 or norm.numel() != 1
          or norm.get_device() != tensors.index):
        raise MagnetonError(N.MAG_E_SIZE, f"norm must be one float32 value on GPU {tensors.index}")
    args = tensors._args(kind, max_norm, eps, norm)
    ws, p, n = _workspace(workspace, lib.mag_clip_gradients_workspace_size, args, tensors.tensors[0])
    _launch(tensors.index, call(lib), args, p, n)
    return norm


def gradient_norm(tensors, *, kind=2, norm=None, workspace=None):
    """The norm of all elements of the tensors together, one float32 value on the GPU
    (`norm`, where it is given).  tensors: float32, float16 and bfloat16 of any shapes (a
    sequence, None left out, or a TensorList), dense or rows of neighbours.  kind: 2, or
    inf for the largest magnitude."""
    return _run(lambda lib: lib.mag_gradient_norm, _list(tensors), kind, 0.0, 0.0, norm, workspace)


def clip_gradients(tensors, max_norm, *, kind=2, eps=1e-6, out=None, norm=None, workspace=None):
    """gradient_norm(), and every tensor times min(1, max_norm / (norm + eps)), in place or
    into `out`: nothing waits for the norm.  An infinite norm makes finite elements zero,
    a norm that is NaN makes all NaN.  Outputs that overlap are refused.  Returns the norm
    before clipping."""
    return _run(lambda lib: lib.mag_clip_gradients, _list(tensors, out), kind, max_norm, eps, norm, workspace)
