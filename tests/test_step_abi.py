"""The norms around a block and the clipping refuse bad arguments on the host, before any
device work (no GPU needed)."""
import ctypes
import math
import os
import random
import subprocess
import sys

import pytest

from test_block_abi import FAKE, NONE, _mat, _n

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
H = _mat(12, 64)
OTHER = _mat(12, 64, data=FAKE + (1 << 20))
ROWS = (FAKE,) * 4


def _forward(N, lib, dtype=2, wdt=0, gdt=0, kind=1, post=0, h=H, y=H, out=H, normed=OTHER, gate=NONE,
             weights=(0, 0, 0, 0), stats=(0, 0, 0, 0), scale=1.0, eps=1e-5):
    return lib.mag_residual_norm(N.RESIDUAL_NORM_ARGS.pack(dtype, wdt, gdt, kind, post, 0, *h, *y, *out, *normed, *gate,
                                                           *weights, *stats, scale, eps), None)


def test_residual_norm_refusals():
    N, lib = _n()
    assert lib.mag_residual_norm(None, None) == N.MAG_E_NULL
    for bad in (dict(dtype=3), dict(wdt=1), dict(kind=2), dict(kind=-1), dict(post=2), dict(y=_mat(12, 63)),
                dict(out=_mat(11, 64)), dict(normed=_mat(12, 64, rs=63)), dict(normed=_mat(12, 64, rs=1, cs=12)),
                dict(h=_mat(12, 0), y=_mat(12, 0), out=_mat(12, 0), normed=_mat(12, 0)), dict(eps=-1.0),
                dict(eps=math.nan), dict(eps=math.inf), dict(scale=math.inf), dict(scale=math.nan),
                dict(weights=(0, 0, FAKE, 0)), dict(weights=(0, 0, 0, FAKE)), dict(gate=_mat(5, 64)),
                dict(gate=_mat(0, 64)), dict(gate=_mat(3, 63)), dict(gate=_mat(3, 64, rs=1, cs=3)),
                dict(gate=_mat(3, 64), gdt=1), dict(out=H, normed=H)):
        assert _forward(N, lib, **bad) == N.MAG_E_SIZE, bad
    for bad in (dict(h=_mat(12, 64, data=0)), dict(y=_mat(12, 64, data=0)), dict(out=_mat(12, 64, data=0))):
        assert _forward(N, lib, **bad) == N.MAG_E_NULL, bad
    for bad in (dict(h=_mat(12, 64, data=FAKE + 1)), dict(weights=(FAKE + 2, 0, 0, 0)), dict(stats=(0, FAKE + 2, 0, 0)),
                dict(gate=_mat(3, 64, data=FAKE + 2))):
        assert _forward(N, lib, **bad) == N.MAG_E_ALIGN, bad
    none = _mat(0, 64)
    assert _forward(N, lib, h=none, y=none, out=none, normed=none) == N.MAG_OK


def _backward(N, lib, dtype=2, wdt=0, gdt=0, kind=1, post=0, h=H, y=H, dn=H, dr=NONE, dh=H, dy=OTHER, gate=NONE,
              dgate=NONE, weights=(0, 0, 0), stats=ROWS, grads=(0, 0, 0, 0), scale=1.0, ws=FAKE, n=1 << 30):
    args = N.RESIDUAL_NORM_BACKWARD_ARGS.pack(dtype, wdt, gdt, kind, post, 0, *h, *y, *dn, *dr, *dh, *dy, *gate, *dgate,
                                              *weights, *stats, *grads, scale)
    return lib.mag_residual_norm_backward(args, ws, n, None)


def test_residual_norm_backward_refusals():
    N, lib = _n()
    assert lib.mag_residual_norm_backward(None, None, 0, None) == N.MAG_E_NULL
    for bad in (dict(dtype=3), dict(kind=2), dict(y=_mat(12, 63)), dict(dn=_mat(11, 64)), dict(dr=_mat(12, 65)),
                dict(dh=_mat(12, 64, rs=63)), dict(scale=math.nan), dict(weights=(0, FAKE, 0)), dict(grads=(0, 0, FAKE, 0)),
                dict(dgate=_mat(1, 64)), dict(gate=_mat(3, 64), dgate=_mat(2, 64)), dict(dh=H, dy=H)):
        assert _backward(N, lib, **bad) == N.MAG_E_SIZE, bad
    for bad in (dict(stats=(0, 0, 0, 0)), dict(kind=0, stats=(0, FAKE, 0, 0)), dict(post=1, stats=(0, FAKE, 0, 0)),
                dict(kind=0, post=1, stats=(FAKE, FAKE, 0, FAKE)), dict(dn=_mat(12, 64, data=0)), dict(ws=0)):
        assert _backward(N, lib, **bad) == N.MAG_E_NULL, bad
    assert _backward(N, lib, n=8) == N.MAG_E_WORKSPACE
    assert _backward(N, lib, ws=FAKE + 8) == N.MAG_E_WORKSPACE
    size = ctypes.c_size_t(0)
    args = N.RESIDUAL_NORM_BACKWARD_ARGS.pack(2, 0, 0, 1, 0, 0, *_mat(300, 4096), *(NONE * 7), *((0,) * 11), 1.0)
    assert lib.mag_residual_norm_backward_workspace_size(args, None) == N.MAG_E_NULL
    assert lib.mag_residual_norm_backward_workspace_size(args, ctypes.byref(size)) == N.MAG_OK
    # column sums of as many workgroups as rows, at most, and four numbers a row
    assert 300 * 5 * 4096 * 4 <= size.value <= 512 * 5 * 4096 * 4 + 300 * 16 + 512


def _tensors(N, lib, refs, kind=0, most=1.0, eps=1e-6, norm=FAKE, n=None, ws=FAKE, bytes_=1 << 30, call="mag_clip_gradients"):
    packed = b"".join(N.TENSOR_REF.pack(*r) for r in refs)
    args = N.TENSORS_ARGS.pack(N.address(packed) if packed else 0, len(refs) if n is None else n, kind, 0, most, eps, norm)
    return getattr(lib, call)(args, ws, bytes_, None)


def _ref(at=0, count=100, cols=0, in_ld=0, out_ld=0, dtype=0, to=None):
    return (FAKE + at, FAKE + (at if to is None else to), count, cols, in_ld, out_ld, dtype, 0)


def test_clip_refusals():
    N, lib = _n()
    assert lib.mag_clip_gradients(None, None, 0, None) == N.MAG_E_NULL
    for bad in (dict(kind=2), dict(most=-1.0), dict(most=math.nan), dict(most=math.inf), dict(eps=-1.0), dict(eps=math.nan),
                dict(n=-1), dict(n=(1 << 16) + 1)):
        assert _tensors(N, lib, [_ref()], **bad) == N.MAG_E_SIZE, bad
    for bad in (_ref(dtype=3), _ref(count=-1), _ref(cols=33), _ref(cols=-1), _ref(cols=10, in_ld=9, out_ld=10),
                _ref(cols=10, in_ld=10, out_ld=(1 << 32) + 1), _ref(to=4), _ref(cols=10, in_ld=10, out_ld=12)):
        assert _tensors(N, lib, [bad]) == N.MAG_E_SIZE, bad
    # the same tensor twice, an output on another's end, columns that share one
    assert _tensors(N, lib, [_ref(), _ref()]) == N.MAG_E_SIZE
    assert _tensors(N, lib, [_ref(), _ref(at=396)]) == N.MAG_E_SIZE
    assert _tensors(N, lib, [_ref(), _ref(at=4000, to=200)]) == N.MAG_E_SIZE
    assert _tensors(N, lib, [_ref(cols=10, in_ld=20, out_ld=20), _ref(at=36, cols=10, in_ld=20, out_ld=20)]) == N.MAG_E_SIZE
    assert _tensors(N, lib, [_ref()], ws=0) == N.MAG_E_NULL
    assert _tensors(N, lib, [_ref()], bytes_=4) == N.MAG_E_WORKSPACE
    assert _tensors(N, lib, [_ref(at=2)]) == N.MAG_E_ALIGN
    assert _tensors(N, lib, [_ref()], norm=FAKE + 2) == N.MAG_E_ALIGN
    assert _tensors(N, lib, [], n=3) == N.MAG_E_NULL
    assert _tensors(N, lib, [(0, 0, 5, 0, 0, 0, 0, 0)]) == N.MAG_E_NULL
    assert _tensors(N, lib, [_ref()], norm=0, call="mag_gradient_norm") == N.MAG_E_NULL
    # nothing to do
    assert _tensors(N, lib, [], norm=0) == N.MAG_OK
    assert _tensors(N, lib, [_ref(count=0)], norm=0) == N.MAG_OK


def test_a_list_made_for_a_call_lives_as_long_as_the_call():
    """the size of a workspace for plain tensors: their description, which the library reads
    by address, must not be freed before (freed memory is overwritten here)"""
    code = """
import paper_2512_08365_amd as mag
from paper_2512_08365_amd import _native as N, _training

def described(n):
    kept = object.__new__(_training.TensorList)
    kept.tensors = kept.out = (None,) * n
    kept._packed = N.TENSOR_REF.pack(4096, 4096, 20000, 0, 0, 0, 2, 0) * n
    return kept

_training._list = described
for n in (1, 2, 40, 300):
    launches = [64] * (n // 64) + [n % 64]
    assert mag.clip_gradients_workspace_size(n) == 8 * sum(min(3 * k, 1024) for k in launches), n
"""
    pytest.importorskip("torch")
    r = subprocess.run([sys.executable, "-c", code], env={**os.environ, "PYTHONMALLOC": "debug"}, cwd=ROOT,
                       capture_output=True, text=True, timeout=120)
    assert r.returncode == 0, r.stdout + r.stderr


def _bytes_of(ref, place, ld):
    _, _, count, cols, *_ = ref
    size = 4 if ref[6] == 0 else 2
    rows = [(place, count)] if cols == 0 else [(place + k * ref[ld] * size, cols) for k in range(count // cols)]
    return {b for at, n in rows for b in range(at, at + n * size)}


def _overlap(refs):
    """whether an output's bytes are another's of the list, byte by byte"""
    out = [_bytes_of(r, r[1], 5) for r in refs]
    own = [r[0] == r[1] and _bytes_of(r, r[0], 4) == o and (r[3] == 0 or r[2] == r[3] or r[4] == r[5])
           for r, o in zip(refs, out)]
    read = [set() if same else _bytes_of(r, r[0], 4) for r, same in zip(refs, own)]
    return any(o & read[j] or (i != j and o & out[j]) for i, o in enumerate(out) for j in range(len(refs)))


def test_tensors_overlap_where_they_share_a_byte_and_nowhere_else():
    """slices of one buffer: columns, rows, single rows, every second row, rows of another
    width, against their bytes one by one"""
    N, lib = _n()

    def refused(refs):
        rc = _tensors(N, lib, refs, bytes_=0)
        assert rc in (N.MAG_E_SIZE, N.MAG_E_WORKSPACE), rc
        return rc == N.MAG_E_SIZE

    def cut(row, rows, col, cols, pitch, step=1):
        return _ref(4 * (row * pitch + col), rows * cols, cols, step * pitch, step * pitch)

    # a row's slice beside other columns, every second row, rows of two pitches
    assert not refused([cut(0, 1, 0, 3, 10), cut(0, 5, 3, 7, 10)])
    assert not refused([_ref(12, 4), cut(0, 5, 7, 3, 10), cut(1, 4, 3, 4, 10)])
    assert not refused([cut(0, 5, 0, 10, 10, 2), cut(1, 5, 0, 10, 10, 2)])
    assert not refused([cut(0, 9, 0, 3, 10), cut(0, 5, 3, 7, 10, 2), cut(1, 4, 3, 7, 10, 2)])
    assert refused([cut(0, 9, 0, 3, 10), cut(1, 4, 2, 7, 10, 2)])
    assert refused([cut(0, 9, 0, 3, 10), cut(8, 1, 2, 1, 10)])
    rng, seen = random.Random(11), [0] * 4
    for _ in range(30000):
        refs = []
        for _ in range(rng.choice((2, 2, 2, 3))):
            cols, dtype = rng.choice((0, 1, 1, 2, 3, 5)), rng.choice((0, 2))
            count = rng.randint(1, 6) * max(cols, 1)
            ld = [cols + rng.choice((0, 1, 2, 7, 12, 31)) for _ in range(2)]
            if rng.random() < 0.7:
                ld[1] = ld[0]
            at = 4 * rng.randint(0, 60)
            to = at if rng.random() < 0.7 else 4 * rng.randint(0, 60)
            refs.append(_ref(at, count, cols, *ld, dtype, to=to))
        want = _overlap(refs)
        seen[want] += 1
        assert refused(refs) == want, refs
    assert min(seen[:2]) > 3000
    # a million rows and some hundred of another pitch among them, which drift past them
    a = (FAKE, FAKE, 3 * 1000003, 3, 7001, 7001, 0, 0)
    for at in range(400):
        start = 4 * (at + 5003 * 7001)
        b = (FAKE + start, FAKE + start, 2 * 580, 2, 7013, 7013, 0, 0)
        meets = any((5003 * 7001 + at + k * 7013 + 1) % 7001 <= 3 and 5003 * 7001 + at + k * 7013 < 1000002 * 7001 + 3
                    for k in range(580))
        assert refused([a, b]) == meets, at
        seen[2 + meets] += 1
    assert min(seen[2:]) > 20
    # rows that no memory holds
    assert _tensors(N, lib, [(FAKE, FAKE, 1 << 36, 1, 1 << 32, 1 << 32, 0, 0)], bytes_=0) == N.MAG_E_SIZE


def test_residual_norm_takes_no_number_that_is_infinite_in_fp32():
    """the kernels take scale and eps as floats"""
    N, lib = _n()
    none = _mat(0, 64)
    for bad in (1e39, -1e39, 3.5e38):
        assert _forward(N, lib, scale=bad) == N.MAG_E_SIZE
        assert _backward(N, lib, scale=bad) == N.MAG_E_SIZE
    assert _forward(N, lib, eps=1e39) == N.MAG_E_SIZE
    for good in (3.4e38, -3.4e38, 0.0):
        assert _forward(N, lib, h=none, y=none, out=none, normed=none, scale=good, eps=abs(good)) == N.MAG_OK
