"""The 8-bit entry points refuse bad arguments on the host, before any device work
(no GPU needed)."""
import ctypes

import pytest

from test_block_abi import FAKE, NONE, _mat, _n, _size


def _quantize(N, lib, dtype=2, fmt=3, block_rows=1, x=_mat(40, 200), q=_mat(40, 200), s=_mat(40, 2), qt=NONE, st=NONE):
    return lib.mag_quantize_fp8(N.QUANTIZE_ARGS.pack(dtype, fmt, block_rows, 0, *x, *q, *s, *qt, *st), None)


def test_quantize_refusals():
    N, lib = _n()
    assert lib.mag_quantize_fp8(None, None) == N.MAG_E_NULL
    assert _quantize(N, lib, dtype=3) == N.MAG_E_SIZE
    assert _quantize(N, lib, fmt=2) == N.MAG_E_SIZE
    assert _quantize(N, lib, fmt=5) == N.MAG_E_SIZE
    for rows in (0, 2, 64, 127, 256, -1):
        assert _quantize(N, lib, block_rows=rows) == N.MAG_E_SIZE
    assert _quantize(N, lib, q=_mat(40, 199)) == N.MAG_E_SIZE
    assert _quantize(N, lib, q=_mat(40, 200, rs=199)) == N.MAG_E_SIZE
    assert _quantize(N, lib, q=_mat(40, 200, rs=1, cs=40)) == N.MAG_E_SIZE
    assert _quantize(N, lib, s=_mat(40, 3)) == N.MAG_E_SIZE
    assert _quantize(N, lib, s=_mat(1, 2)) == N.MAG_E_SIZE
    assert _quantize(N, lib, block_rows=128) == N.MAG_E_SIZE
    assert _quantize(N, lib, s=_mat(40, 2, rs=1)) == N.MAG_E_SIZE          # lines overlap
    assert _quantize(N, lib, s=_mat(40, 2, rs=1, cs=39)) == N.MAG_E_SIZE
    assert _quantize(N, lib, s=_mat(40, 2, rs=2, cs=100)) == N.MAG_E_SIZE
    assert _quantize(N, lib, s=_mat(40, 2, data=FAKE + 2)) == N.MAG_E_ALIGN
    assert _quantize(N, lib, s=_mat(40, 2, data=0)) == N.MAG_E_NULL
    assert _quantize(N, lib, x=_mat(40, 200, data=0)) == N.MAG_E_NULL
    assert _quantize(N, lib, x=_mat(40, 200, data=FAKE + 1)) == N.MAG_E_ALIGN
    assert _quantize(N, lib, x=_mat(40, 200, rs=-1)) == N.MAG_E_SIZE
    assert _quantize(N, lib, qt=_mat(40, 200), st=_mat(40, 2)) == N.MAG_E_SIZE
    assert _quantize(N, lib, qt=_mat(200, 40), st=_mat(200, 2)) == N.MAG_E_SIZE
    # nothing to write
    assert _quantize(N, lib, q=NONE) == N.MAG_OK
    assert _quantize(N, lib, x=_mat(0, 200), q=_mat(0, 200), s=_mat(0, 2)) == N.MAG_OK
    assert _quantize(N, lib, x=_mat(40, 0), q=_mat(40, 0), s=_mat(40, 0)) == N.MAG_OK


def _linear(N, lib, dtype=2, act=0, fx=3, fw=3, x=_mat(40, 200), w=_mat(64, 200), res=NONE, pre=NONE, y=_mat(40, 64),
            sx=_mat(40, 2), sw=_mat(1, 2), bias=0, ws=FAKE, n=1 << 30):
    return lib.mag_linear_fp8(N.LINEAR_FP8_ARGS.pack(dtype, act, fx, fw, *x, *w, *res, *pre, *y, *sx, *sw, bias), ws, n,
                              None)


def test_linear_refusals():
    N, lib = _n()
    assert lib.mag_linear_fp8(None, None, 0, None) == N.MAG_E_NULL
    for dtype in (0, 3, -1):
        assert _linear(N, lib, dtype=dtype) == N.MAG_E_SIZE
    assert _linear(N, lib, act=5) == N.MAG_E_SIZE
    assert _linear(N, lib, fx=2) == N.MAG_E_SIZE
    assert _linear(N, lib, fw=5) == N.MAG_E_SIZE
    assert _linear(N, lib, w=_mat(64, 201)) == N.MAG_E_SIZE
    assert _linear(N, lib, y=_mat(40, 63)) == N.MAG_E_SIZE
    assert _linear(N, lib, y=_mat(40, 64, rs=63)) == N.MAG_E_SIZE
    assert _linear(N, lib, res=_mat(40, 63)) == N.MAG_E_SIZE
    assert _linear(N, lib, pre=_mat(39, 64)) == N.MAG_E_SIZE
    assert _linear(N, lib, sx=_mat(40, 1)) == N.MAG_E_SIZE
    assert _linear(N, lib, sx=_mat(1, 2)) == N.MAG_E_SIZE
    assert _linear(N, lib, sx=NONE) == N.MAG_E_SIZE
    assert _linear(N, lib, sw=_mat(2, 2)) == N.MAG_E_SIZE
    assert _linear(N, lib, sw=_mat(64, 3)) == N.MAG_E_SIZE
    assert _linear(N, lib, sx=_mat(40, 2, rs=(1 << 22) + 1)) == N.MAG_E_SIZE
    assert _linear(N, lib, sx=_mat(40, 2, data=FAKE + 2)) == N.MAG_E_ALIGN
    assert _linear(N, lib, sw=_mat(1, 2, data=0)) == N.MAG_E_NULL
    assert _linear(N, lib, x=_mat(40, 200, data=0)) == N.MAG_E_NULL
    assert _linear(N, lib, w=_mat(64, 200, data=0)) == N.MAG_E_NULL
    assert _linear(N, lib, y=_mat(40, 64, data=FAKE + 1)) == N.MAG_E_ALIGN
    assert _linear(N, lib, bias=FAKE + 1) == N.MAG_E_ALIGN
    big = (1 << 21) + 1
    assert _linear(N, lib, w=_mat(big, 200), y=_mat(40, big)) == N.MAG_E_SIZE
    assert _linear(N, lib, x=_mat(0, 200), y=_mat(0, 64), sx=_mat(0, 2)) == N.MAG_OK
    assert _linear(N, lib, w=_mat(0, 200), y=_mat(40, 0), sw=_mat(0, 2)) == N.MAG_OK


def test_linear_workspace():
    N, lib = _n()

    def size(x, w):
        return _size(lib.mag_linear_fp8_workspace_size,
                     N.LINEAR_FP8_ARGS.pack(2, 0, 3, 3, *x, *w, *NONE, *NONE, *NONE, *NONE, *NONE, 0))

    assert lib.mag_linear_fp8_workspace_size(None, ctypes.byref(ctypes.c_size_t(0))) == N.MAG_E_NULL
    # rows of whole 16 bytes are read where they lie, others are packed first
    rc, plain = size(_mat(4000, 208), _mat(6400, 208))
    assert rc == N.MAG_OK and plain == 0
    for x, w in ((_mat(4000, 200), _mat(6400, 208, rs=208)), (_mat(4000, 208, data=FAKE + 8), _mat(6400, 208)),
                 (_mat(4000, 208), _mat(6400, 208, rs=1, cs=6400))):
        w = (*w[:2], x[2], *w[3:])
        rc, n = size(x, w)
        assert rc == N.MAG_OK and n > 0
        assert _linear(N, lib, x=x, w=w, y=_mat(4000, 6400), sx=_mat(4000, 2), sw=_mat(50, 2), n=n - 1) == N.MAG_E_WORKSPACE
        assert _linear(N, lib, x=x, w=w, y=_mat(4000, 6400), sx=_mat(4000, 2), sw=_mat(50, 2), ws=None) == N.MAG_E_NULL
        assert _linear(N, lib, x=x, w=w, y=_mat(4000, 6400), sx=_mat(4000, 2), sw=_mat(50, 2),
                       ws=FAKE + 16) == N.MAG_E_WORKSPACE
    # few rows are read as they lie
    assert size(_mat(8, 200), _mat(64, 200)) == (N.MAG_OK, 0)


def test_binding_refusals():
    torch = pytest.importorskip("torch")
    import paper_2512_08365_amd as mag
    x = torch.ones(4, 16)
    q = x.to(torch.float8_e4m3fn)
    for call in (lambda: mag.quantize_fp8(x), lambda: mag.linear_fp8(q, x, q, x),
                 lambda: mag.linear_fp8_workspace_size(q, q)):
        with pytest.raises(mag.MagnetonError) as e:
            call()
        assert e.value.code == -1
