"""Which kernels the calls that share, add up and evict enqueue, and that each launch has fewer than 2^32 threads at the largest sizes that the
header allows.  Launches are noted on the host and none is enqueued."""
import json
import os
import subprocess
import sys

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
    log.launch_log_start(-1, 0)
    if c["entry"] == "evict":
        rc = lib.approxifer_cache_evict(at, at, at, at, c["stride"], at, at, at, 2, c["heads"][1], 256, c["B"], c["M"], c["P"], c["page"], c["budget"],
                                        0, 0, at, 1 << 62, None)
    else:
        seq = binding._Sequences(at, at, at, c["T"], c["B"], c["M"], c["P"], c["page"])
        Hq, Hkv, Dh = c["heads"]
        size, q, ws = (Hq, Hkv, Dh, c["dtype"]), (at, Hq * Dh, at, at, at), c["workspace"]
        length, tail = c.get("length", c["M"] * c["page"]), (c.get("window", 0), 0, 1.0, at, at)
        if c["entry"] == "mass":
            rc = lib.approxifer_attend_mass(seq, *size, *q, at, length, c["rows"], length, *tail, ws, None)
        else:
            rc = lib.approxifer_attend_shared(seq, *size, *q, at, at, c["C"], c["rows"], length, c["shared"], *tail, ws, None)
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
    got = [json.loads(line) for line in r.stdout.splitlines()]
    assert len(got) == len(calls)
    for c, (rc, launches) in zip(calls, got):
        assert rc == 0 and launches, c
        for name, *threads in launches:
            assert all(0 < int(n) < 1 << 32 for n in threads), (c, name, threads)
    return [[n[0] for n in launches] for _, launches in got]


def _kinds(names):
    return [k for n in names for k in ("shared_both", "shared_tiles", "shared_tokens", "shared_join", "attend_scores", "attend_join", "attend_tiles",
                                       "attend_tokens", "attend_mass", "add_slices", "mass_of_scores", "evict_select", "evict_pages", "evict_move")
            if k in n]


BASE = dict(M=1 << 26, P=1 << 30, page=16, workspace=1 << 62)


def test_every_launch_fits(tmp_path):
    calls = []
    for dtype in (0, 1, 2):
        for B, heads in ((1 << 20, (4, 4, 64)), (1 << 20, (8, 4, 64)), (1 << 19, (64, 8, 8)), (4096, (1024, 1024, 64)), (1 << 20, (4, 1, 256)),
                         (1 << 20, (1, 1, 128)), (1, (64, 8, 128)), (700, (64, 8, 128)), (700, (1024, 1, 128))):
            group = heads[0] // heads[1]
            T = min(1 << 24, (1 << 30) // heads[0])
            for rows in {1, *(-(-n // group) for n in (16, 17, 33, 64, 65, 129)), T}:
                call = dict(BASE, T=T, B=B, heads=heads, dtype=dtype, rows=rows)
                calls += [dict(call, entry="mass"), dict(call, entry="mass", workspace=1 << 33)]
                calls += [dict(call, entry="shared", C=C, shared=1 << 29) for C in {1, min(B, 100), max(1, B // 2)}]
    for B in (1, 1 << 20):
        calls += [dict(BASE, entry="evict", B=B, heads=(8, 8, 128), stride=stride, budget=budget) for stride in (100, 1 << 30)
                  for budget in (1, 1 << 30)]
    _launches(tmp_path, calls)


def test_which_kernels_have_a_call(tmp_path):
    def shared(B=192, T=192, rows=1, C=1, heads=(32, 8, 128), dtype=2, shared=8000, length=8500, workspace=1 << 40, **f):
        return dict(dict(BASE, entry="shared", B=B, T=T, rows=rows, C=C, heads=heads, dtype=dtype, shared=shared, length=length, workspace=workspace), **f)

    def mass(B=16, T=16, rows=1, heads=(32, 8, 128), dtype=2, length=30000, workspace=1 << 40):
        return dict(BASE, entry="mass", B=B, T=T, rows=rows, heads=heads, dtype=dtype, length=length, workspace=workspace)

    calls = {
        "both in one": (shared(), ["shared_both", "shared_join"]),
        "no such instance": (shared(heads=(32, 8, 96)), ["shared_tiles", "shared_tokens", "shared_join"]),
        "small pages": (shared(page=8), ["shared_tiles", "shared_tokens", "shared_join"]),
        "few rows": (shared(B=24, T=24, heads=(12, 12, 64), dtype=0), ["shared_tokens", "shared_join"]),
        "several rows each": (shared(T=960, rows=5), ["shared_tiles", "shared_join"]),
        "rows that fill a tile": (shared(T=192 * 128, rows=128), ["attend_tiles"]),
        "hardly two a group": (shared(C=100), ["attend_tokens"]),
        "nothing shared": (shared(shared=0), ["attend_tokens"]),
        "no workspace": (shared(workspace=0), ["attend_tokens"]),
        "scores kept": (mass(), ["attend_scores", "attend_join", "mass_of_scores"]),
        "scores kept, whole": (mass(B=600, T=600, length=200), ["attend_scores", "mass_of_scores"]),
        "many rows": (mass(B=2, T=8000, rows=4000, length=4000), ["attend_tiles", "attend_mass", "add_slices"]),
        "statistics alone": (mass(workspace=16 * 32 * 8), ["attend_tokens", "attend_mass"]),
        "too many scores": (mass(B=1000, T=1000, length=100000), ["attend_tokens", "attend_mass"]),
    }
    got = _launches(tmp_path, [c for c, _ in calls.values()])
    for (name, (_, want)), names in zip(calls.items(), got):
        assert _kinds(names) == want, (name, names)
    assert _kinds(_launches(tmp_path, [dict(BASE, entry="evict", B=3, heads=(8, 8, 128), stride=5000, budget=100)])[0]) == [
        "evict_select", "evict_pages", "evict_move"]
