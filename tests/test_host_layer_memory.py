"""The entry points for the layers around a product where the host has no memory: on the stand-in for the HIP runtime, every allocation of a call fails in
turn.  The call returns DMM_ENOMEM, or does without; nothing passes a C entry, and the next call is as if there had been none before."""
import ctypes
import os
import shutil
import subprocess
import sys

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
if ROOT not in sys.path:
    sys.path.insert(0, ROOT)

from tests.test_host_calls import Recorder, recorder  # noqa: E402, F401
from tests.test_host_layer import Space, made  # noqa: E402


def run(rec, new, which):
    from paper_2510_08874_amd import binding as b
    for layout, m, k, n in (("whole", 40, 4096, 300), ("uneven", 1301, 1103, 907), ("row_col", 9, 2000, 12001)):
        d = made(layout, m, k, n)
        s = Space(True)
        a, w, v = s.integers(d[0], "rows"), s.integers(d[1], "cols"), s.integers(d[1], "cols")
        t = [s.tiles(x, 2)[0] for x in (d[0], d[1], d[1], d[2], d[2], d[2], d[2], d[2], d[2], d[0], d[1], d[1])]
        x, desc = s.tiles(d[0], 2)[0], b.matrix_desc(d[0])
        forms = s.integers(d[0], "rows"), s.integers(d[0], "cols")
        call = {"int_quantize": lambda p: b.dmm_int_quantize(desc, b.DMM_BF16, x, *forms), "int_dequantize": lambda p: b.dmm_int_dequantize(desc, forms[1], b.DMM_MX_COLS, b.DMM_BF16, x),
                "int_execute": lambda p: p.execute_int(a, w, t[3], b.DMM_C_BF16, 0), "int_gated_execute": lambda p: p.gated_int(b.DMM_SILU, a, w, v, t[3], 0),
                "gated_execute": lambda p: p.gated(b.DMM_SILU, *t[:6], 0), "gated_backward": lambda p: p.gated_backward(b.DMM_SILU, *t[:3], *t[4:12], 0, 0),
                "execute_backward": lambda p: p.execute_backward(t[0], t[1], t[3], t[9], t[10], 0, 0)}[which]
        plan = b.Plan(*d, 12)
        at = len(rec.ops())
        call(plan)
        want = [(o[1], rec.so.rec_blocks(o[0])) for o in rec.launches(at)]
        fails = 0
        for after in list(range(60)) + [100, 300, 1000]:
            plan = b.Plan(*d, 12)
            new.new_fails_after(after)
            try:
                call(plan)
            except b.DmmError as e:
                assert e.kind == "ENOMEM", e
                fails += 1
            failed = new.new_has_failed()
            new.new_fails_after(-1)
            at = len(rec.ops())
            call(plan)
            assert [(o[1], rec.so.rec_blocks(o[0])) for o in rec.launches(at)] == want, (layout, after)
            plan.destroy()
            if not failed:
                break
        assert fails, layout


CALLS = ["int_quantize", "int_dequantize", "int_execute", "int_gated_execute", "gated_execute", "gated_backward", "execute_backward"]


@pytest.fixture(scope="session")
def no_memory(tmp_path_factory):
    if shutil.which("g++") is None:
        pytest.skip("needs g++")
    so = str(tmp_path_factory.mktemp("no_memory") / "no_memory.so")
    subprocess.run(["g++", "-std=c++17", "-O1", "-shared", "-fPIC", os.path.join(ROOT, "tests", "native", "no_memory.cpp"), "-o", so], check=True, capture_output=True, text=True)
    return so


@pytest.mark.parametrize("which", CALLS)
def test_no_memory(recorder, no_memory, which):  # noqa: F811
    run = subprocess.run([sys.executable, os.path.abspath(__file__), recorder, no_memory, which], capture_output=True, text=True, cwd=ROOT, timeout=300)
    assert run.returncode == 0, run.stdout[-2000:] + run.stderr[-4000:]


if __name__ == "__main__":
    new = ctypes.CDLL(sys.argv[2], mode=ctypes.RTLD_GLOBAL)
    run(Recorder(sys.argv[1]), new, sys.argv[3])
