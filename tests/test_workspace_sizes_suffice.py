"""With a workspace of the size that is asked for, attention's calls launch what they do with any larger one.  Launches are noted on the host and
none is enqueued."""
import json
import os
import subprocess
import sys

import pytest

import launch_log

_RUN = r"""
import json, sys, ctypes
sys.path[:0] = sys.argv[3:5]
log = ctypes.CDLL(sys.argv[1], mode=ctypes.RTLD_GLOBAL)
log.launch_log.restype = ctypes.c_char_p
from paper_2109_09868_amd import binding
binding.LIB_PATH = sys.argv[2]
lib, at = binding.load(), 1 << 20
for line in sys.stdin:
    c = json.loads(line)
    T, B, rows, length, window, sinks = c["T"], c["B"], c["rows"], c["length"], c["window"], c["sinks"]
    size = (*c["heads"], c["dtype"])
    if c["entry"] == "shared":
        need = lib.approxifer_attend_shared_workspace_bytes(T, B, c["C"], *size, rows, length, c["shared"], window, sinks)
    else:
        need = getattr(lib, "approxifer_%s_workspace_bytes" % c["entry"])(T, B, *size, rows, length, window, sinks)
    got = []
    for workspace in (need, 1 << 62):
        log.launch_log_start(-1, 0)
        seq = binding._Sequences(at, at, at, T, B, -(-length // c["page"]), 1 << 30, c["page"])
        q, tail = (at, size[0] * size[2], at, at, at), (window, sinks, 1.0, at, at if workspace else None, workspace, None)
        if c["entry"] == "attend":
            rc = lib.approxifer_attend(seq, *size, *q, rows, length, *tail)
        elif c["entry"] == "attend_mass":
            rc = lib.approxifer_attend_mass(seq, *size, *q, at, length, rows, length, *tail)
        else:
            rc = lib.approxifer_attend_shared(seq, *size, *q, at, at, c["C"], rows, length, c["shared"], *tail)
        got.append([rc, log.launch_log().decode().splitlines()])
    print(json.dumps([need, got]))
"""


def _launches(folder, calls):
    """[(bytes asked for, launches with as many, launches with any number), ..]; a launch: its kernel and its grid."""
    from paper_2109_09868_amd import build
    name = 'log_ += names()[host] + "\\n";'
    assert name in launch_log.SHIM
    each = 'log_ += names()[host]; for (uint32_t n : {grid.x, grid.y, grid.z}) log_ += " " + std::to_string(n); log_ += "\\n";'
    src, shim = str(folder / "grids.cpp"), str(folder / "libgrids.so")
    with open(src, "w") as f:
        f.write(launch_log.SHIM.replace(name, each))
    subprocess.run([build.host_compiler(), "-O1", "-std=c++17", "-fPIC", "-shared", src, "-o", shim, "-ldl"], check=True)
    here = os.path.dirname(os.path.abspath(__file__))
    r = subprocess.run([sys.executable, "-c", _RUN, shim, launch_log.library_path(), here, os.path.dirname(here)], text=True,
                       input="".join(json.dumps(c) + "\n" for c in calls), capture_output=True, timeout=100)
    assert r.returncode == 0, r.stderr
    got = [json.loads(line) for line in r.stdout.splitlines()]
    assert len(got) == len(calls)
    assert all(rc == 0 for _, both in got for rc, _ in both)
    return [(need, a, b) for need, ((_, a), (_, b)) in got]


@pytest.mark.parametrize("entry", ["attend", "attend_mass", "attend_shared"])
def test_the_size_that_is_asked_for_is_enough(tmp_path, entry):
    calls = []
    for dtype in (0, 1, 2):
        for heads in ((8, 8, 128), (32, 8, 128), (12, 12, 64), (8, 1, 256), (6, 2, 40), (1, 1, 64)):
            for B, rows in ((1, 1), (1, 5), (1, 300), (3, 1), (16, 1), (16, 7), (32, 1), (64, 2), (4, 150), (700, 1)):
                for length, window, sinks in ((60, 0, 0), (700, 0, 0), (4000, 0, 0), (8192, 0, 0), (131072, 0, 0), (40000, 4096, 4)):
                    call = dict(entry=entry, T=B * rows, B=B, rows=rows, heads=heads, dtype=dtype, length=length, window=window, sinks=sinks, page=16)
                    if entry == "attend_shared":
                        calls += [dict(call, entry="shared", C=C, shared=length * 3 // 4) for C in {1, max(1, B // 8)}]
                    else:
                        calls.append(call)
    several = 0
    for call, (need, asked, any_number) in zip(calls, _launches(tmp_path, calls)):
        assert asked == any_number, (call, need)
        several += any("join" in line for line in asked)
    assert several > len(calls) // 10
