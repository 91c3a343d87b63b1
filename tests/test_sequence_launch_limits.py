"""Every launch of the cached-sequence calls at the largest sizes that the header allows has fewer than 2^32 threads, which is what the
runtime takes.  Launches are noted on the host and none is enqueued."""
import json
import os
import subprocess
import sys

import launch_log

_RUN = r"""
import ctypes, json, sys
sys.path[:0] = sys.argv[3:5]
log = ctypes.CDLL(sys.argv[1], mode=ctypes.RTLD_GLOBAL)
log.launch_log.restype = ctypes.c_char_p
from paper_2109_09868_amd import binding
binding.LIB_PATH = sys.argv[2]
lib, at = binding.load(), 1 << 20
for line in sys.stdin:
    c = json.loads(line)
    seq = binding._Sequences(at, at, at, c["T"], c["B"], c["M"], c["P"], c["page"])
    Hq, Hkv, Dh = c["heads"]
    log.launch_log_start(-1, 0)
    if c["entry"] == "append":
        freq = (ctypes.c_double * 4)(1.0, 0.5, 0.25, 0.1)
        q = at + c["odd"]
        rc = lib.approxifer_append(seq, Hq, Hkv, Dh, c["dtype"], q, Hq * Dh, at, Hkv * Dh, at, Hkv * Dh, at, at, at, at, at, 1e-6, None, 1,
                                   freq, None, 4, 0, at, None)
    elif c["entry"] == "attend":
        rc = lib.approxifer_attend(seq, Hq, Hkv, Dh, c["dtype"], at, Hq * Dh, at, at, at, c["rows"], c["M"] * c["page"], 0, 0, 1.0, at, at,
                                   c["workspace"], None)
    elif c["entry"] == "reserve":
        rc = lib.approxifer_cache_reserve(at, at, at, at, at, c["B"], c["M"], c["P"], c["page"], None)
    elif c["entry"] == "fork":
        rc = lib.approxifer_cache_fork(at, at, at, at, at, at, at, at, at, at, 2, 4096, c["B"], c["B"], c["M"], c["P"], c["page"], at, 1 << 60, None)
    else:
        rc = lib.approxifer_cache_compact(at, at, at, at, at, at, 2, 4096, c["B"], c["M"], c["P"], c["page"], at, 1 << 60, None)
    print(json.dumps([rc, [l.split() for l in log.launch_log().decode().splitlines()]]))
"""


def _launches(folder, calls):
    """[(return code, [(kernel, threads in x, y, z), ..]), ..]"""
    from paper_2109_09868_amd import build
    name = 'log_ += names()[host] + "\\n";'
    assert name in launch_log.SHIM
    each = 'log_ += names()[host]; for (uint64_t n : {uint64_t(grid.x) * block.x, uint64_t(grid.y) * block.y, uint64_t(grid.z) * block.z}) ' \
           'log_ += " " + std::to_string(n); log_ += "\\n";'
    src, shim = str(folder / "launches.cpp"), str(folder / "liblaunches.so")
    with open(src, "w") as f:
        f.write(launch_log.SHIM.replace(name, each))
    subprocess.run([build.host_compiler(), "-O1", "-std=c++17", "-fPIC", "-shared", src, "-o", shim, "-ldl"], check=True)
    here = os.path.dirname(os.path.abspath(__file__))
    r = subprocess.run([sys.executable, "-c", _RUN, shim, launch_log.library_path(), here, os.path.dirname(here)], text=True,
                       input="".join(json.dumps(c) + "\n" for c in calls), capture_output=True, timeout=100)
    assert r.returncode == 0, r.stderr
    return [json.loads(line) for line in r.stdout.splitlines()]


def _check(folder, calls):
    got = _launches(folder, calls)
    assert len(got) == len(calls)
    for c, (rc, launches) in zip(calls, got):
        assert rc == 0 and launches, c
        for name, *threads in launches:
            assert all(0 < int(n) < 1 << 32 for n in threads), (c, name, threads)
    return got


def test_attention(tmp_path):
    calls = []
    for dtype in (0, 1, 2):
        for B, heads in ((1 << 20, (4, 4, 64)), (1 << 20, (8, 4, 64)), (1 << 19, (64, 8, 8)), (4096, (1024, 1024, 64)), (1 << 20, (4, 1, 256)),
                         (1 << 20, (1, 1, 128)), (1, (64, 8, 128)), (700, (64, 8, 128))):
            group = heads[0] // heads[1]
            T = min(1 << 24, (1 << 30) // heads[0])
            for rows in {1, *(-(-n // group) for n in (16, 17, 33, 48, 49, 64, 65, 128, 129)), T}:
                for workspace in (0, 1 << 40):
                    calls.append(dict(entry="attend", T=T, B=B, M=1 << 26, P=1 << 30, page=16, heads=heads, dtype=dtype, rows=rows,
                                      workspace=workspace))
    got = _check(tmp_path, calls)
    names = {"tiles" if "attend_tiles" in n[0] else "tokens" for _, launches in got for n in launches if "join" not in n[0]}
    assert names == {"tiles", "tokens"}


def test_append_and_pages(tmp_path):
    base = dict(T=1 << 24, B=1 << 20, M=1 << 26, P=1 << 30, page=16, heads=(4, 4, 64), dtype=2, odd=0)
    calls = [dict(base, entry="append", odd=odd, dtype=dtype, heads=heads, T=min(1 << 24, (1 << 30) // heads[0]), B=min(1 << 20, (1 << 22) // heads[1]))
             for odd in (0, 4) for dtype in (0, 2) for heads in ((4, 4, 64), (64, 1, 8), (1024, 1024, 256), (64, 64, 128))]
    calls += [dict(base, entry=e, P=P, B=B) for e in ("reserve", "fork", "compact") for P in (1, 1 << 30) for B in (1, 1 << 20)]
    _check(tmp_path, calls)
