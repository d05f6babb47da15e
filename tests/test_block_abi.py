"""The block operators' entry points refuse bad arguments on the host, before
any device work (no GPU needed)."""
import ctypes
import math

import pytest

FAKE = 4096


def _n():
    from paper_2512_08365_amd import _native as N
    return N, N.load()


def _mat(rows, cols, data=FAKE, rs=None, cs=1):
    return (data, rows, cols, cols if rs is None else rs, cs)


NONE = (0, 0, 0, 0, 0)


def _size(call, args):
    b = ctypes.c_size_t(0)
    return call(args, ctypes.byref(b)), b.value


def _linear(N, lib, dtype=1, act=0, x=_mat(4, 16), w=_mat(8, 16), res=NONE, pre=NONE,
            y=_mat(4, 8), bias=0, ws=None, n=0):
    return lib.mag_linear(N.LINEAR_ARGS.pack(dtype, act, *x, *w, *res, *pre, *y, bias), ws, n, None)


def test_linear_refusals():
    N, lib = _n()
    assert lib.mag_linear(None, None, 0, None) == N.MAG_E_NULL
    assert _linear(N, lib, dtype=3) == N.MAG_E_SIZE
    assert b"dtype" in lib.mag_last_error()
    assert _linear(N, lib, act=5) == N.MAG_E_SIZE
    assert _linear(N, lib, act=-1) == N.MAG_E_SIZE
    assert _linear(N, lib, w=_mat(8, 15)) == N.MAG_E_SIZE
    assert _linear(N, lib, y=_mat(4, 9)) == N.MAG_E_SIZE
    assert _linear(N, lib, y=_mat(3, 8)) == N.MAG_E_SIZE
    assert _linear(N, lib, res=_mat(4, 9)) == N.MAG_E_SIZE
    assert _linear(N, lib, pre=_mat(5, 8)) == N.MAG_E_SIZE
    assert _linear(N, lib, y=_mat(4, 8, cs=4, rs=1)) == N.MAG_E_SIZE
    assert _linear(N, lib, y=_mat(4, 8, rs=7)) == N.MAG_E_SIZE
    assert _linear(N, lib, pre=_mat(4, 8, rs=0)) == N.MAG_E_SIZE
    assert _linear(N, lib, x=_mat(-1, 16), y=_mat(-1, 8)) == N.MAG_E_SIZE
    assert _linear(N, lib, x=_mat(4, 16, rs=-16)) == N.MAG_E_SIZE
    assert _linear(N, lib, x=_mat(4, 16, rs=(1 << 32) + 1)) == N.MAG_E_SIZE
    big = N.MAG_MAX_EXTENT + 1
    assert _linear(N, lib, x=_mat(big, 16), y=_mat(big, 8)) == N.MAG_E_SIZE
    assert _linear(N, lib, x=_mat(4, 16, data=0)) == N.MAG_E_NULL
    assert _linear(N, lib, w=_mat(8, 16, data=0)) == N.MAG_E_NULL
    assert _linear(N, lib, y=_mat(4, 8, data=0)) == N.MAG_E_NULL
    assert _linear(N, lib, x=_mat(4, 16, data=FAKE + 1)) == N.MAG_E_ALIGN
    assert _linear(N, lib, dtype=0, y=_mat(4, 8, data=FAKE + 2)) == N.MAG_E_ALIGN
    assert _linear(N, lib, bias=FAKE + 1) == N.MAG_E_ALIGN
    # nothing to write: nothing is launched
    assert _linear(N, lib, x=_mat(0, 16), y=_mat(0, 8)) == N.MAG_OK
    assert _linear(N, lib, w=_mat(0, 16), y=_mat(4, 0)) == N.MAG_OK


def test_linear_workspace():
    N, lib = _n()
    b = ctypes.c_size_t(0)
    args = N.LINEAR_ARGS.pack(0, 0, *_mat(300, 77), *_mat(130, 77), *NONE, *NONE, *NONE, 0)
    assert lib.mag_linear_workspace_size(args, None) == N.MAG_E_NULL
    assert lib.mag_linear_workspace_size(None, ctypes.byref(b)) == N.MAG_E_NULL
    rc, size = _size(lib.mag_linear_workspace_size, args)
    assert rc == N.MAG_OK
    if size:
        def call(ws, n):
            return _linear(N, lib, dtype=0, x=_mat(300, 77), w=_mat(130, 77), y=_mat(300, 130),
                           ws=ws, n=n)

        assert call(None, size) == N.MAG_E_NULL
        assert call(FAKE + 8, size) == N.MAG_E_WORKSPACE
        assert call(FAKE, size - 1) == N.MAG_E_WORKSPACE


def _backward(N, lib, dtype=1, act=0, x=_mat(40, 16), w=_mat(8, 16), pre=NONE, dy=_mat(40, 8),
              dx=_mat(40, 16), dw=_mat(8, 16), db=FAKE, ws=FAKE, n=0):
    return lib.mag_linear_backward(
        N.LINEAR_BACKWARD_ARGS.pack(dtype, act, *x, *w, *pre, *dy, *dx, *dw, db), ws, n, None)


def test_linear_backward_refusals():
    N, lib = _n()
    assert lib.mag_linear_backward(None, None, 0, None) == N.MAG_E_NULL
    big = 1 << 30
    assert _backward(N, lib, dtype=-1, n=big) == N.MAG_E_SIZE
    assert _backward(N, lib, act=7, n=big) == N.MAG_E_SIZE
    assert _backward(N, lib, dy=_mat(40, 9), n=big) == N.MAG_E_SIZE
    assert _backward(N, lib, dx=_mat(40, 15), n=big) == N.MAG_E_SIZE
    assert _backward(N, lib, dw=_mat(9, 16), n=big) == N.MAG_E_SIZE
    assert _backward(N, lib, dw=_mat(8, 16, rs=1, cs=8), n=big) == N.MAG_E_SIZE
    assert _backward(N, lib, act=2, n=big) == N.MAG_E_SIZE  # no pre
    assert _backward(N, lib, act=2, pre=_mat(40, 8, data=0), n=big) == N.MAG_E_NULL
    assert _backward(N, lib, dy=_mat(40, 8, data=0), n=big) == N.MAG_E_NULL
    assert _backward(N, lib, w=_mat(8, 16, data=0), n=big) == N.MAG_E_NULL
    assert _backward(N, lib, db=FAKE + 1, n=big) == N.MAG_E_ALIGN
    rc, size = _size(lib.mag_linear_backward_workspace_size,
                     N.LINEAR_BACKWARD_ARGS.pack(1, 0, *_mat(40, 16), *_mat(8, 16), *NONE,
                                                 *_mat(40, 8), *NONE, *NONE, 0))
    assert rc == N.MAG_OK and size > 0
    assert _backward(N, lib, n=size - 1) == N.MAG_E_WORKSPACE
    assert _backward(N, lib, ws=FAKE + 128, n=size) == N.MAG_E_WORKSPACE
    assert _backward(N, lib, ws=None, n=size) == N.MAG_E_NULL


def _norm(N, dtype=1, wt=0, x=_mat(4, 16), y=_mat(4, 16), dy=NONE, dx=NONE, w=0, b=0, mean=0,
          rstd=0, dw=0, db=0, eps=1e-5):
    return N.NORM_ARGS.pack(dtype, wt, *x, *y, *dy, *dx, w, b, mean, rstd, dw, db, eps)


def test_layer_norm_refusals():
    N, lib = _n()
    f = lib.mag_layer_norm
    assert f(None, None) == N.MAG_E_NULL
    assert f(_norm(N, dtype=4), None) == N.MAG_E_SIZE
    assert f(_norm(N, dtype=1, wt=2), None) == N.MAG_E_SIZE
    assert f(_norm(N, x=_mat(4, 0), y=_mat(4, 0)), None) == N.MAG_E_SIZE
    assert f(_norm(N, y=_mat(4, 15)), None) == N.MAG_E_SIZE
    assert f(_norm(N, y=_mat(4, 16, rs=8)), None) == N.MAG_E_SIZE
    for eps in (-1e-9, math.inf, math.nan):
        assert f(_norm(N, eps=eps), None) == N.MAG_E_SIZE
    assert f(_norm(N, x=_mat(4, 16, data=0)), None) == N.MAG_E_NULL
    assert f(_norm(N, w=FAKE + 2), None) == N.MAG_E_ALIGN
    assert f(_norm(N, mean=FAKE + 1), None) == N.MAG_E_ALIGN
    assert f(_norm(N, x=_mat(0, 16), y=_mat(0, 16)), None) == N.MAG_OK


def test_layer_norm_backward_refusals():
    N, lib = _n()
    rc, size = _size(lib.mag_layer_norm_backward_workspace_size, _norm(N))
    assert rc == N.MAG_OK

    def f(**kw):
        kw = {"y": NONE, "dy": _mat(4, 16), "dx": _mat(4, 16), "mean": FAKE, "rstd": FAKE,
              "dw": FAKE, "db": FAKE, **kw}
        return lib.mag_layer_norm_backward(_norm(N, **kw), FAKE, 1 << 30, None)

    assert lib.mag_layer_norm_backward(None, None, 0, None) == N.MAG_E_NULL
    assert f(dy=_mat(4, 15)) == N.MAG_E_SIZE
    assert f(dx=_mat(3, 16)) == N.MAG_E_SIZE
    assert f(mean=0) == N.MAG_E_NULL
    assert f(rstd=0) == N.MAG_E_NULL
    assert f(rstd=FAKE + 2) == N.MAG_E_ALIGN
    assert f(dw=FAKE + 2) == N.MAG_E_ALIGN
    assert f(dy=_mat(4, 16, data=0)) == N.MAG_E_NULL


def _orth(N, dtype=0, steps=5, batch=1, g=_mat(32, 48), out=_mat(32, 48), gb=0, ob=0, a=3.4445,
          b=-4.775, c=2.0315, eps=1e-7):
    return N.ORTHOGONALIZE_ARGS.pack(dtype, steps, batch, *g, *out, gb, ob, a, b, c, eps)


def test_orthogonalize_refusals():
    N, lib = _n()
    rc, size = _size(lib.mag_orthogonalize_workspace_size, _orth(N))
    assert rc == N.MAG_OK and size > 0

    def f(ws=FAKE, n=1 << 30, **kw):
        return lib.mag_orthogonalize(_orth(N, **kw), ws, n, None)

    assert lib.mag_orthogonalize(None, None, 0, None) == N.MAG_E_NULL
    assert f(dtype=9) == N.MAG_E_SIZE
    assert f(steps=-1) == N.MAG_E_SIZE
    assert f(steps=N.MAG_ORTH_MAX_STEPS + 1) == N.MAG_E_SIZE
    assert f(batch=-1) == N.MAG_E_SIZE
    assert f(out=_mat(48, 32)) == N.MAG_E_SIZE
    assert f(batch=2, gb=32 * 48, ob=32 * 48 - 1) == N.MAG_E_SIZE  # overlap
    assert f(a=math.nan) == N.MAG_E_SIZE
    assert f(eps=-1.0) == N.MAG_E_SIZE
    assert f(a=1e5, steps=20) == N.MAG_E_SIZE  # grows past any float
    assert f(g=_mat(32, 48, data=0)) == N.MAG_E_NULL
    assert f(n=size - 1) == N.MAG_E_WORKSPACE
    assert f(ws=FAKE + 4) == N.MAG_E_WORKSPACE
    assert f(batch=0) == N.MAG_OK
    assert f(g=_mat(0, 48), out=_mat(0, 48)) == N.MAG_OK


def test_binding_refuses_cpu_tensors():
    torch = pytest.importorskip("torch")
    import paper_2512_08365_amd as mag
    x = torch.ones(4, 16)
    for call in (lambda: mag.linear(x, x), lambda: mag.layer_norm(x),
                 lambda: mag.orthogonalize(x), lambda: mag.linear_backward(x, x, x),
                 lambda: mag.layer_norm_backward(x, x, x[:, 0], x[:, 0])):
        with pytest.raises(mag.MagnetonError) as e:
            call()
        assert e.value.code == -1
