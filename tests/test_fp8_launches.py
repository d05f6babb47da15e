"""What the 8-bit linear layer launches, for which sizes: its host code over launches
that are only written down (fp8_launches.cpp), so no GPU is needed and no kernel runs."""
import ctypes
import os
import subprocess

import pytest

HERE = os.path.dirname(os.path.abspath(__file__))
ROOT = os.path.dirname(HERE)
X, WEIGHT, Y, X_SCALE, W_SCALE, WORK = (k << 56 for k in range(1, 7))
NONE = (0, 0, 0, 0, 0)
SIDE = (64, 128, 256)
BF16, E4M3 = 2, 3


class Calls:
    def __init__(self, so):
        from paper_2512_08365_amd import _build, _native
        self.N = _native
        subprocess.check_call([_build.hipcc(), "-x", "hip", "--cuda-host-only", "-std=c++17", "-O1",
                               "-fPIC", "-shared", "-I", os.path.join(ROOT, "include"), "-o", so,
                               os.path.join(HERE, "fp8_launches.cpp")])
        self.lib = ctypes.CDLL(so)
        self.lib.launches.restype = self.lib.last_error.restype = ctypes.c_char_p

    def linear(self, x, weight, by_row=False):
        """(launches, bytes of workspace)"""
        rows, inner, outer = x[1], x[2], weight[1]
        blocks, n = -(-inner // 128), ctypes.c_size_t(0)
        tall = outer if by_row else -(-outer // 128)
        args = self.N.LINEAR_FP8_ARGS.pack(BF16, 0, E4M3, E4M3, *x, *weight, *NONE, *NONE, Y, rows, outer, outer, 1,
                                           X_SCALE, rows, blocks, 1, rows, W_SCALE, tall, blocks, 1, tall, 0)
        assert self.lib.mag_linear_fp8_workspace_size(args, ctypes.byref(n)) == 0, self.lib.last_error()
        self.lib.clear_launches()
        rc = self.lib.mag_linear_fp8(args, ctypes.c_void_p(WORK), n, None)
        assert rc == 0, (rc, self.lib.last_error())
        return [{k: v if k == "what" else int(v) for k, v in (f.split("=") for f in line.split())}
                for line in self.lib.launches().decode().splitlines()], n.value


@pytest.fixture(scope="module")
def calls(tmp_path_factory):
    return Calls(str(tmp_path_factory.mktemp("launches") / "fp8_launches.so"))


def _rows(data, rows, cols, pitch):
    return (data, rows, cols, pitch, 1)


INNER = [1, 15, 16, 127, 1000, 4096, (1 << 23) - 256, (1 << 23) - 129, (1 << 23) - 128, (1 << 23) - 16, 1 << 23,
         (1 << 23) + 1, (1 << 23) + 65536, 9_000_000, 11_200_000, 17_000_001, 50_000_000, (1 << 30) - 8, 1 << 30]
SIZES = [(33, 1), (64, 64), (33, 1 << 21), (300, 70), (1024, 1024), (2048, 2048), (1 << 21, 33)]


@pytest.mark.parametrize("rows,outer", SIZES)
def test_offsets_inside_a_tile_stay_below_31_bits(calls, rows, outer):
    """a load's offset from its tile's first byte has 31 bits; beyond them lie zeros.  What a
    product reads is the operand or what was packed for it, all of the reduction, once"""
    for inner in INNER:
        lays = [lambda d, n: _rows(d, n, inner, -(-inner // 16) * 16), lambda d, n: _rows(d, n, inner, inner + 1),
                lambda d, n: (d, n, inner, 1, n), lambda d, n: _rows(d, n, inner, 1), lambda d, n: _rows(d, n, inner, 0)]
        for lx in lays:
            for lw in (lays if inner >= 1 << 22 else lays[:3]):
                x, w = lx(X, rows), lw(WEIGHT, outer)
                for by_row in (False, True):
                    launches, size = calls.linear(x, w, by_row)
                    _check(launches, size, x, w, by_row)


def _check(launches, size, x, w, by_row):
    case = (x, w, by_row)
    rows, inner, outer = x[1], x[2], w[1]
    packed = {}
    done, planes, joined = 0, 0, False
    for p in launches:
        if p["what"] == "pack":
            of = X if p["src"] < WEIGHT else WEIGHT
            m = x if of == X else w
            # (from the reduction's next part on)
            assert p["src"] == of + done * (m[4] if inner > 1 else 0) and p["rows"] == m[1], case
            assert WORK <= p["dst"] and p["dst"] + p["rows"] * p["ld"] <= WORK + size and p["ld"] >= p["cols"], case
            packed[of] = p
        elif p["what"] == "tiles":
            for o, ld, n, of, m in (("a", "lda", rows, X, x), ("b", "ldb", outer, WEIGHT, w)):
                reach = (min(SIDE[p["tile"]], n) - 1) * p[ld] + 128
                assert reach < (1 << 31) - 16, (case, p)
                if of in packed:
                    q = packed[of]
                    assert p[o] == q["dst"] and p[ld] == q["ld"] and q["cols"] == p["K"], (case, p)
                else:
                    assert p[o] == of + done and (n == 1 or p[ld] == m[3]) and p[ld] % 16 == 0, (case, p)
            assert done % 128 == 0
            assert p["sa"] == X_SCALE + done // 128 * p["sa_cs"] * 4, (case, p)
            assert p["sb"] == W_SCALE + done // 128 * p["sb_cs"] * 4, (case, p)
            done += p["K"]
            if p["dtype"] == 0:
                plane = p["R"] * p["partial_ld"] * 4
                if planes == 0:
                    first = p["partial"]
                assert p["partial"] == first + planes * plane and p["partial_ld"] >= outer, (case, p)
                planes += p["splits"]
                assert WORK <= first and first + planes * plane <= WORK + size, (case, p)
                for q in packed.values():
                    assert first >= q["dst"] + q["rows"] * q["ld"], (case, p)
            else:
                assert p["dtype"] == BF16 and p["splits"] == 1, (case, p)
        else:
            assert p["what"] == "join" and p["splits"] == planes and p["partial"] == first, (case, p)
            joined = True
    assert done == inner and joined == (planes > 0), (case, launches)
    if len(packed) == 2:
        a, b = (packed[k] for k in (X, WEIGHT))
        assert a["dst"] + a["rows"] * a["ld"] <= b["dst"], case
