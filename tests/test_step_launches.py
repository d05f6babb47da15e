"""The launches of the norms around a block and of quantization: the library's host code in
a child process over the stand-in runtime (hip_double.c), which writes them down (no GPU
needed)."""
import ctypes
import importlib.util
import os
import re
import subprocess
import sys

HERE = os.path.dirname(os.path.abspath(__file__))
ROOT = os.path.dirname(HERE)
FAKE = 4096
NONE = (0, 0, 0, 0, 0)


def _native():
    # (without the package, which would bring another library's kernels along)
    spec = importlib.util.spec_from_file_location(
        "native", os.path.join(ROOT, "paper_2512_08365_amd", "_native.py"))
    N = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(N)
    lib = N.load()
    log = ctypes.CDLL(None)
    log.double_log.restype = ctypes.c_char_p

    def launches():
        lines = [x.split() for x in log.double_log().decode().splitlines()]
        return [(x[1], int(x[3]), int(x[5])) for x in lines if x[0] == "launch"]

    return N, lib, log, launches


def _threads_of_a_row():
    """a workgroup's threads hold a row of eight elements each, also where there are no
    rows: each thread leaves its columns' sums"""
    N, lib, log, launches = _native()
    for width in (8, 300, 512, 513, 1024, 1025, 2048, 2049, 2056, 4096, 4097, 8192):
        for groups, each in ((1, 0), (3, 0), (3, 1), (3, 2), (1, 70), (600, 1), (600, 2)):
            x, gate = (FAKE, groups * each, width, width, 1), (FAKE, groups, width, width, 1)
            for dtype in (0, 1, 2):
                log.double_clear()
                args = N.RESIDUAL_NORM_BACKWARD_ARGS.pack(
                    dtype, 0, 0, 1, 1, 0, *x, *x, *x, *NONE, *x, *NONE, *gate, *gate, *[FAKE] * 11, 1.0)
                assert lib.mag_residual_norm_backward(args, 256, 1 << 40, None) == 0
                back = [x for x in launches() if "k_residual_norm_back" in x[0]]
                assert len(back) == 1 and back[0][2] * 8 >= width, (width, groups, each, back)


def _workgroups_of_quantization():
    """all rows have their workgroups, and no launch 2^32 threads"""
    N, lib, log, launches = _native()
    for rows, cols in ((1, 1), (1000, 700), ((1 << 28) - 16, 128), (1 << 28, 1), ((1 << 28) + 1, 513), (1 << 30, 100),
                       (1 << 30, 5000), (1 << 23, 100_000), (3, 1 << 30)):
        m, n = -(-rows // 128), -(-cols // 128)
        for by_columns in (False, True):
            x = (FAKE, rows, cols, 1, rows) if by_columns else (FAKE, rows, cols, cols, 1)
            q, qt = (FAKE, rows, cols, cols, 1), (FAKE, cols, rows, rows, 1)
            for block_rows in (1, 128):
                s = (FAKE, rows if block_rows == 1 else m, n, 1, 1 << 30)
                st = (FAKE, cols if block_rows == 1 else n, m, 1, 1 << 30)
                for outputs in ((q, s, NONE, NONE), (q, s, qt, st), (NONE, NONE, qt, st)):
                    log.double_clear()
                    rc = lib.mag_quantize_fp8(N.QUANTIZE_ARGS.pack(2, 3, block_rows, 0, *x, *outputs[0], *outputs[1],
                                                                   *outputs[2], *outputs[3]), None)
                    assert rc == 0, (rows, cols, by_columns, lib.mag_last_error())
                    made = launches()
                    for name, grid, block in made:
                        assert 0 < grid * block < 1 << 32, (rows, cols, made)
                    whole = sum(grid for _, grid, _ in made)
                    if "k_quantize_rows" in made[0][0]:
                        r, c = (cols, rows) if by_columns and cols > 1 else (rows, cols)
                        assert whole == -(-r // 16) * -(-(-(-c // 128)) // 4), (rows, cols, made)
                    else:
                        assert whole == m * n, (rows, cols, made)


def _child(tmp_path, name):
    so = str(tmp_path / "hip_double.so")
    subprocess.check_call(["gcc", "-O1", "-shared", "-fPIC", "-o", so, os.path.join(HERE, "hip_double.c")])
    env = dict(os.environ)
    env["LD_PRELOAD"] = " ".join(x for x in (env.get("LD_PRELOAD"), so) if x)
    r = subprocess.run([sys.executable, os.path.abspath(__file__), name], env=env, capture_output=True, text=True,
                       timeout=120)
    assert r.returncode == 0, r.stdout + r.stderr


def test_workgroups_of_the_backward_pass_hold_their_rows(tmp_path):
    _child(tmp_path, "_threads_of_a_row")


def test_workgroups_of_quantization_fit_their_launches(tmp_path):
    _child(tmp_path, "_workgroups_of_quantization")


def test_the_stand_in_runtime_has_a_place_for_every_kernel():
    """(it leaves those beyond its table without a name)"""
    from paper_2512_08365_amd import _native
    with open(os.path.join(HERE, "hip_double.c")) as f:
        places = int(re.search(r"g_fns\[(\d+)\];", f.read()).group(1))
    symbols = subprocess.check_output(["nm", _native.LIB_PATH], text=True)
    assert 0 < symbols.count("__device_stub__") <= places


if __name__ == "__main__":
    globals()[sys.argv[1]]()
