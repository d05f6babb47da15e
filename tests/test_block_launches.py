"""What the feed-forward block's calls launch, for which sizes: their host code
over launches that are only written down (block_launches.cpp), so no GPU is
needed and no kernel runs."""
import ctypes
import math
import os
import random
import subprocess

import block_sizes
import pytest

HERE = os.path.dirname(os.path.abspath(__file__))
ROOT = os.path.dirname(HERE)
FAKE = 1 << 20
NONE = (0, 0, 0, 0, 0)
F32, F16, BF16 = 0, 1, 2
# products: bfloat16, half, fp32, fp32 in three parts, an update's two halves
K_BF16, K_F16, K_F32, K_PARTS, K_HALVES = range(5)
SIDE = (64, 128, 256)


class Calls:
    def __init__(self, so):
        from paper_2512_08365_amd import _build, _native
        self.N = _native
        subprocess.check_call([_build.hipcc(), "-x", "hip", "--cuda-host-only", "-std=c++17", "-O1",
                               "-fPIC", "-shared", "-I", os.path.join(ROOT, "include"), "-o", so,
                               os.path.join(HERE, "block_launches.cpp")])
        self.lib = ctypes.CDLL(so)
        self.lib.launches.restype = self.lib.last_error.restype = ctypes.c_char_p

    def _call(self, name, args):
        n = ctypes.c_size_t(0)
        assert getattr(self.lib, f"mag_{name}_workspace_size")(args, ctypes.byref(n)) == 0, \
            self.lib.last_error()
        self.lib.clear_launches()
        rc = getattr(self.lib, f"mag_{name}")(args, ctypes.c_void_p(FAKE), n, None)
        assert rc == 0, (rc, self.lib.last_error())
        return [{k: v if k == "what" else float(v) if k in ("scale", "mix", "diagonal") else int(v)
                 for k, v in (f.split("=") for f in line.split())}
                for line in self.lib.launches().decode().splitlines()]

    def linear(self, dtype, x, weight):
        y = _rows(x[1], weight[1])
        return self._call("linear", self.N.LINEAR_ARGS.pack(dtype, 0, *x, *weight, *NONE, *NONE, *y, 0))

    def linear_backward(self, dtype, x, weight, dy):
        return self._call("linear_backward", self.N.LINEAR_BACKWARD_ARGS.pack(
            dtype, 0, *x, *weight, *NONE, *dy, *_rows(x[1], x[2]), *_rows(weight[1], x[2]), FAKE))

    def orthogonalize(self, dtype, rows, cols, steps=5, batch=1, coefficients=(3.4445, -4.775, 2.0315)):
        m = _rows(rows, cols)
        return self._call("orthogonalize", self.N.ORTHOGONALIZE_ARGS.pack(
            dtype, steps, batch, *m, *m, rows * cols, rows * cols, *coefficients, 1e-7))


@pytest.fixture(scope="module")
def calls(tmp_path_factory):
    return Calls(str(tmp_path_factory.mktemp("launches") / "block_launches.so"))


def _rows(rows, cols, gap=0):
    return (FAKE, rows, cols, cols + gap, 1)


def _columns(rows, cols, gap=0):
    return (FAKE, rows, cols, 1, rows + gap)


def _products(launches):
    return [p for p in launches if p["what"] in ("linear", "partial", "two", "update")]


def _reach(p, o):
    """bytes from a tile's first one to the end of what its loads read of operand o"""
    parts = {K_PARTS: 3, K_HALVES: 2}.get(p["kind"], 1)
    size = 4 if p["kind"] == K_F32 else 2
    step = 64 if p["kind"] in (K_BF16, K_F16) else 32
    side = SIDE[p["tile"]]
    if p[f"{o}_mc"]:
        lines, line = min(step, p["K"]), side * parts * size
    else:
        lines, line = min(side, p["R" if o == "a" else "S"]), step * parts * size
    return (lines - 1) * p[f"{o}_ld"] * size + line


ROWS = [40, 3_000_000, 3_000_001, 4_194_304, 4_300_000, 8_400_001, 11_600_000, 17_100_000, 20_000_000,
        35_000_000, (1 << 30) - 8, 1 << 30]
FEATURES = [(8, 8), (64, 16), (65, 70), (512, 512), (4096, 257), (257, 4096), (1 << 21, 8), (8, 1 << 21)]


@pytest.mark.parametrize("dtype", [F32, F16, BF16])
@pytest.mark.parametrize("lay", [_rows, _columns])
def test_offsets_inside_a_tile_stay_below_31_bits(calls, lay, dtype):
    """a load's offset from its tile's first byte has 31 bits; beyond them lie zeros"""
    for rows in ROWS:
        for inner, outer in FEATURES:
            for gap in (0, 3):
                x, dy = lay(rows, inner, gap), lay(rows, outer, gap)
                for w in (_rows(outer, inner, gap), _columns(outer, inner, gap)):
                    for p in _products(calls.linear(dtype, x, w) + calls.linear_backward(dtype, x, w, dy)):
                        for o in ("a", "b"):
                            assert _reach(p, o) < (1 << 31) - 16, (rows, inner, outer, gap, p)


@pytest.mark.parametrize("rows,cols", [(8, 1 << 21), (1 << 21, 8), (1 << 21, 3000), (3000, 1 << 21)])
def test_offsets_of_long_updates_stay_below_31_bits(calls, rows, cols):
    for dtype in (F32, F16, BF16):
        for p in _products(calls.orthogonalize(dtype, rows, cols)):
            for o in ("a", "b"):
                assert _reach(p, o) < (1 << 31) - 16, p


@pytest.mark.parametrize("dtype", [F32, F16, BF16])
@pytest.mark.parametrize("size", [(40, 72), (96, 6000), (700, 100)])
def test_scales_of_polynomials_that_contract_are_finite(calls, size, dtype):
    """bounds that fall to zero, at once or step by step, beside ones that grow"""
    rng = random.Random(7)
    drawn = [tuple(rng.choice((-1, 1)) * 10 ** rng.uniform(-30, e) for e in (2, 1, 1)) for _ in range(50)]
    for coefficients in [(0, 0, 0), (1e-200, 0, 0), (0.1, 0, 0), (1e-3, 1e-3, 0), (1e-160, 1e-160, 1e-160),
                         (0.5, -0.25, 0.1), (2, -1.5, 0.5), (1.5, 0, 0), *drawn]:
        for steps in (1, 2, 3, 8, 64):
            try:
                launches = calls.orthogonalize(dtype, *size, steps, 2, coefficients)
            except AssertionError:
                assert b"grows" in calls.lib.last_error()
                continue
            for p in launches:
                if p["what"] == "begin":
                    assert 0 < p["scale"] < math.inf
                elif p["what"] in ("update", "partial"):
                    assert all(math.isfinite(p[k]) for k in ("scale", "mix", "diagonal")), (coefficients, p)


def test_spans_beyond_63_bits_of_bytes_are_refused(calls):
    """2^30 rows 2^32 elements apart are 2^64 bytes of fp32"""
    N, lib = calls.N, calls.lib
    size = ctypes.c_size_t(0)

    def linear(x):
        return lib.mag_linear_workspace_size(
            N.LINEAR_ARGS.pack(F32, 0, *x, *_rows(8, x[2]), *NONE, *NONE, *NONE, 0), ctypes.byref(size))

    assert linear((FAKE, 1 << 30, 16, 1 << 32, 1)) == N.MAG_E_SIZE and b"2^60" in lib.last_error()
    assert linear((FAKE, 1 << 28, 1 << 21, 1 << 32, 1 << 32)) == N.MAG_E_SIZE
    assert linear((FAKE, 1 << 28, 16, 1 << 31, 1)) == 0
    assert linear((FAKE, 1, 16, 1 << 62, 1)) == 0   # (one row: its stride may be anything)

    def update(batch, g_stride, out_stride):
        m = _rows(8, 16)
        return lib.mag_orthogonalize(N.ORTHOGONALIZE_ARGS.pack(
            F32, 5, batch, *m, *m, g_stride, out_stride, 2.0, -1.5, 0.5, 1e-7), ctypes.c_void_p(FAKE),
            ctypes.c_size_t(1 << 40), None)

    assert update(2, 128, 128) == 0 and update(2, 0, 1 << 40) == 0
    for g_stride, out_stride in (((1 << 60) // 2 + 1, 128), (128, (1 << 60) // 2 + 1), (128, 1 << 62)):
        assert update(2, g_stride, out_stride) == N.MAG_E_SIZE, (g_stride, out_stride)


def _variant(p):
    """what a product is compiled for: its result, kind, tile, steps in LDS, operands across"""
    side, steps = SIDE[p["tile"]], 2 if p["tile"] else 4
    if side == 128 and p["what"] in ("linear", "update") and p["kind"] != K_PARTS:
        tr, ts = -(-p["R"] // 128), -(-p["S"] // 128)
        units = (tr * (tr + 1) // 2 if p["symmetric"] else tr * ts) * p["batch"]
        steps = 4 if units <= 256 and p["K"] >= 32 * (64 if p["kind"] in (K_BF16, K_F16) else 32) else 2
    return p["what"], p["kind"], side, steps, p["a_mc"], p["b_mc"]


def test_the_sizes_of_the_gpu_tests_reach_every_variant(calls):
    """a change of the costs that a tile is chosen by must not leave one untested"""
    types = {"f32": F32, "f16": F16, "bf16": BF16}
    reached = set()
    for ty, dtype in types.items():
        for rows, inner, outer in block_sizes.LINEAR[ty]:
            for lx in (_rows, _columns):
                for lw in (_rows, _columns):
                    reached |= {_variant(p) for p in _products(calls.linear(
                        dtype, lx(rows, inner), lw(outer, inner)))}
        for rows, inner, outer in block_sizes.LINEAR_BACKWARD[ty]:
            reached |= {_variant(p) for p in _products(calls.linear_backward(
                dtype, _rows(rows, inner), _rows(outer, inner), _rows(rows, outer)))}
    for batch, rows, cols in block_sizes.UPDATES:
        for dtype in types.values():
            reached |= {_variant(p) for p in _products(calls.orthogonalize(dtype, rows, cols, batch=batch))}
    every = [(a, b) for a in (0, 1) for b in (0, 1)]
    want = set()
    for kind in (K_BF16, K_F16):
        want |= {("linear", kind, *tile, *ab) for tile in ((64, 4), (128, 2), (128, 4), (256, 2)) for ab in every}
        want |= {("partial", kind, *tile, *ab) for tile in ((64, 4), (128, 2)) for ab in every}
    want |= {(what, K_F32, 64, 4, *ab) for what in ("linear", "partial") for ab in every}
    want |= {(what, K_PARTS, *tile, *ab) for what in ("linear", "partial") for tile in ((64, 4), (128, 2))
             for ab in every}
    want |= {("two", kind, 64, 4, a, 1) for kind in (K_BF16, K_F16, K_F32, K_PARTS) for a in (0, 1)}
    # an update's X X^T takes both operands alike, its long product X across or neither
    want |= {("partial", K_HALVES, *tile, a, a) for tile in ((64, 4), (128, 2)) for a in (0, 1)}
    want |= {("update", K_HALVES, *tile, *ab) for tile in ((64, 4), (128, 2), (128, 4), (256, 2))
             for ab in ((0, 0), (0, 1), (1, 1))}
    assert want - reached == set()
    assert reached - want == set()


@pytest.mark.parametrize("size,steps,_", block_sizes.GROUPED)
def test_sizes_that_take_several_steps_at_once(calls, size, steps, _):
    """fewer long products than steps, for two-byte results alone"""
    for dtype in (F32, F16, BF16):
        long = [p for p in _products(calls.orthogonalize(dtype, *size, steps)) if not p["symmetric"]]
        assert len(long) == steps if dtype == F32 else len(long) < steps, (dtype, len(long))
