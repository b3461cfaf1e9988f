"""What appending and the block norm launch for any number of tokens, without a GPU: grids stay within the limits of a launch (fewer than 2^32 threads along
x) and hold every token."""
import json
import os
import subprocess
import sys

import paper_2601_11676_amd as H

HERE = os.path.dirname(os.path.abspath(__file__))

CALLS = """
import ctypes as C, json, sys
recorder = C.CDLL(sys.argv[1], mode=C.RTLD_GLOBAL)
recorder.recorder_take.restype = C.c_char_p
lib = C.CDLL(sys.argv[2])
p, i64, out = C.c_void_p(1 << 30), C.c_int64, []
for what, n, d, dtype in json.load(sys.stdin):
    if what == "norm":
        rc = lib.halo_block_norm(p, p, None, None, None, p, p, n, d, dtype, dtype, 1, 0, C.c_float(1.0), C.c_float(1e-5), None)
    else:
        shape = C.byref((C.c_int32 * 7)(d, d, 16, 16, 1000, 4, dtype))
        q = C.c_void_p(1 << 31)
        rc = lib.halo_paged_append(shape, n, p, i64(d * 16), p, i64(d * 16), p, i64(d * 16), p, None if what == "append" else p, 1000, p, None, 0, 0, 0,
                                   q, p, p, None)
    out.append((rc, [l.split() for l in recorder.recorder_take().decode().split("\\n")[:-1]]))
json.dump(out, sys.stdout)
"""


def test_grids_of_any_number_of_tokens(tmp_path):
    shim, top = str(tmp_path / "recorder.so"), (1 << 31) - 1
    subprocess.run(["gcc", "-O1", "-shared", "-fPIC", "-o", shim, os.path.join(HERE, "launch_recorder.c")], check=True)
    calls = [(what, n, d, dtype) for what, d in (("norm", 8), ("norm", 512), ("norm", 520), ("norm", 8192), ("norm", 32768), ("append", 1), ("listed", 8))
             for n in (1, 5, 1 << 22, (1 << 24) - 1, 1 << 24, (1 << 26) - 4, 1 << 26, top) for dtype in (0, 1)]
    p = subprocess.run([sys.executable, "-c", CALLS, shim, H.library_path()], input=json.dumps(calls), capture_output=True, text=True, timeout=120)
    assert p.returncode == 0, p.stderr
    for (what, n, d, dtype), (rc, launches) in zip(calls, json.loads(p.stdout)):
        assert rc == 0, (what, n, d)
        rows_a_group = 4 if what == "norm" and d <= 512 else 1
        groups = [int(x) for _, x, _, _, _ in launches]
        threads = int(launches[0][4])
        assert sum(groups) == -(-n // rows_a_group), (what, n, d, launches)
        # as few launches as there can be, up to a workgroup each
        assert len(launches) == -(-sum(groups) // (((1 << 32) - 1) // threads)), (what, n, d, launches)
        assert len({tuple(x[4:]) + tuple(x[2:4]) + (x[0],) for x in launches}) == 1
