"""The launches of the feed-forward block's norms: the library's host code in a
child process over the stand-in runtime (hip_double.c), which writes them down."""
import ctypes
import importlib.util
import os
import subprocess
import sys

HERE = os.path.dirname(os.path.abspath(__file__))
ROOT = os.path.dirname(HERE)
FAKE = 4096


def _child():
    # (without the package, which would bring another library's kernels along)
    spec = importlib.util.spec_from_file_location(
        "native", os.path.join(ROOT, "paper_2512_08365_amd", "_native.py"))
    N = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(N)
    lib = N.load()
    log = ctypes.CDLL(None)
    log.double_log.restype = ctypes.c_char_p
    for rows in (1, 70_000, (1 << 22) - 1, 1 << 22, 1 << 30):
        for cols, lay in ((8, (1, rows)), (1, (1, 7)), (20_000, (20_000, 1)), (8, (8, 1))):
            m, out = (FAKE, rows, cols, *lay), (FAKE, rows, cols, cols, 1)
            for dtype in (0, 1, 2):
                log.double_clear()
                args = N.NORM_ARGS.pack(dtype, dtype, *m, *out, *m, *out, *[FAKE] * 6, 1e-5)
                assert lib.mag_layer_norm(args, None) == 0
                assert lib.mag_layer_norm_backward(args, FAKE, 1 << 40, None) == 0
                lines = [x.split() for x in log.double_log().decode().splitlines()]
                launches = [(x[1], int(x[3]), int(x[5])) for x in lines if x[0] == "launch"]
                assert len(launches) >= 3
                for name, grid, block in launches:
                    assert 0 < grid * block < 1 << 32, (rows, cols, name, grid, block)
                # one column is a row like any other, whatever its stride
                wide = cols == 20_000 or (cols == 8 and lay[1] != 1)
                assert any("k_norm_wide" in x[0] for x in launches) == wide, launches
                assert any("k_norm_back_wide" in x[0] for x in launches) == wide, launches


def test_launches_stay_below_32_bits_of_threads(tmp_path):
    so = str(tmp_path / "hip_double.so")
    subprocess.check_call(["gcc", "-O1", "-shared", "-fPIC", "-o", so, os.path.join(HERE, "hip_double.c")])
    env = dict(os.environ)
    env["LD_PRELOAD"] = " ".join(x for x in (env.get("LD_PRELOAD"), so) if x)
    r = subprocess.run([sys.executable, os.path.abspath(__file__)], env=env, capture_output=True, text=True,
                       timeout=120)
    assert r.returncode == 0, r.stdout + r.stderr


if __name__ == "__main__":
    _child()
