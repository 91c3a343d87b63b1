"""What the calls on a cache that add up, share and evict decide on the host, without a GPU: codes, refusals, sizes."""
import ctypes
import os

import pytest

from paper_2109_09868_amd import binding

FAKE = ctypes.c_void_p(4096)                                  # never dereferenced: every call below ends before a launch
ODD = ctypes.c_void_p(4097)


@pytest.fixture(scope="module")
def lib():
    if not os.path.exists(binding.LIB_PATH):
        import __graft_entry__
        __graft_entry__.build()
    return binding.load()


def _evict(lib, table=FAKE, lens=FAKE, refs=FAKE, mass=FAKE, stride=64, kept=FAKE, status=FAKE, pools=FAKE, planes=2, heads=2, row=128,
           B=2, M=3, P=5, page=16, budget=20, first=1, recent=3, ws=FAKE, ws_bytes=1 << 20):
    return lib.approxifer_cache_evict(table, lens, refs, mass, stride, kept, status, pools, planes, heads, row, B, M, P, page, budget, first,
                                      recent, ws, ws_bytes, None)


def test_evict_refusals(lib):
    for missing in ("table", "lens", "refs", "mass", "kept", "pools"):
        assert _evict(lib, **{missing: None}) == -1, missing
    for bad in (dict(stride=-1), dict(planes=-1), dict(heads=-1), dict(row=-16), dict(budget=0), dict(budget=-5), dict(first=-1),
                dict(recent=-1), dict(first=21), dict(first=18, recent=3), dict(recent=1 << 62, first=1 << 62), dict(budget=1 << 62, recent=1 << 63)):
        if bad.get("recent", 0) >= 1 << 63:
            bad = dict(bad, recent=-(1 << 63))
        assert _evict(lib, **bad) == -2, bad
    for bad in (dict(B=-1), dict(M=0), dict(P=0), dict(page=0), dict(page=12)):
        assert _evict(lib, **bad) == -11, bad
    for bad in (dict(B=(1 << 20) + 1), dict(M=1 << 28), dict(P=(1 << 30) + 1), dict(page=8192), dict(budget=(1 << 30) + 1), dict(heads=1025),
                dict(row=1040), dict(planes=(1 << 20) + 1)):
        assert _evict(lib, **bad) == -3, bad
    for bad in (dict(pools=ODD), dict(row=24), dict(row=8), dict(ws=ODD)):
        assert _evict(lib, **bad) == -10, bad
    need = binding.approxifer_cache_evict_workspace_bytes(2, 20, 5, 16)
    assert _evict(lib, ws=None) == -12 and _evict(lib, ws_bytes=need - 1) == -12 and need >= 4 * (2 * 20 + 2 * 2 + 5)
    assert _evict(lib, B=0, table=None, lens=None, mass=None, kept=None, ws=None) == 0
    for none in ((0, 20, 5, 16), (2, 0, 5, 16), (2, 20, 0, 16), (2, 20, 5, 12), (2, 1 << 31, 5, 16)):
        assert binding.approxifer_cache_evict_workspace_bytes(*none) == 0


def _seq(T=4, B=2, M=3, P=5, page=16, table=4096, lens=4096, starts=4096):
    return binding._Sequences(table, lens, starts, T, B, M, P, page)


def _mass(lib, seq=None, Hq=4, Hkv=2, Dh=64, dtype=0, q=FAKE, qs=256, kp=FAKE, vp=FAKE, out=FAKE, mass=FAKE, stride=48, rows=1, length=48,
          window=0, sinks=0, scale=1.0, status=FAKE, ws=FAKE, ws_bytes=256):
    s = ctypes.byref(seq if seq is not None else _seq()) if seq is not False else None
    return lib.approxifer_attend_mass(s, Hq, Hkv, Dh, dtype, q, qs, kp, vp, out, mass, stride, rows, length, window, sinks, scale, status, ws,
                                      ws_bytes, None)


def _sizes_are_refused(lib, call):
    for bad in (dict(T=-1), dict(B=-1), dict(M=0), dict(P=0), dict(page=0), dict(page=24), dict(page=-16)):
        assert call(lib, _seq(**bad)) == -11, bad
    for bad in (dict(T=(1 << 24) + 1), dict(B=(1 << 20) + 1), dict(P=1 << 31), dict(M=1 << 28), dict(page=8192)):
        assert call(lib, _seq(**bad)) == -3, bad
    for bad in (dict(Hq=0), dict(Hkv=0), dict(Hq=3), dict(Dh=0), dict(Dh=-8), dict(Dh=60)):
        assert call(lib, **bad) == -11, bad
    assert call(lib, Hq=2048, qs=2048 * 64) == -3 and call(lib, Dh=264, qs=4 * 264) == -3
    for dtype in (-1, 3, 7):
        assert call(lib, dtype=dtype) == -9
    assert call(lib, False) == -1
    for missing in ("table", "lens", "starts"):
        assert call(lib, _seq(**{missing: None})) == -1
    assert call(lib, _seq(B=0)) == -11
    assert call(lib, _seq(B=0, T=0, table=None, lens=None, starts=None)) == 0
    assert call(lib, _seq(T=0), status=None) == 0
    for missing in ("q", "kp", "vp", "out"):
        assert call(lib, **{missing: None}) == -1
    for bad in (dict(rows=-1), dict(length=-1), dict(window=-1), dict(sinks=-1), dict(scale=float("nan")), dict(scale=float("inf")),
                dict(qs=255)):
        assert call(lib, **bad) == -2, bad
    for odd in ("q", "kp", "vp", "out", "ws"):
        assert call(lib, **{odd: ODD}) == -10


def test_attend_mass_refusals(lib):
    _sizes_are_refused(lib, _mass)
    assert _mass(lib, mass=None) == -1 and _mass(lib, mass=ODD) == -10 and _mass(lib, stride=-1) == -2
    assert _mass(lib, ws=None) == -12 and _mass(lib, ws_bytes=255) == -12
    import torch
    need = binding.approxifer_attend_mass_workspace_bytes
    for args in ((0, 2, 4, 2, 64), (4, 0, 4, 2, 64), (4, 2, 3, 2, 64), (4, 2, 4, 2, 60), (4, 2, 4, 2, 264)):
        assert need(*args, torch.float16, 1, 100) == 0
    assert need(4, 2, 4, 2, 64, torch.float16, 1, 100) >= 256


def _shared(lib, seq=None, Hq=4, Hkv=2, Dh=64, dtype=0, q=FAKE, qs=256, kp=FAKE, vp=FAKE, out=FAKE, groups=FAKE, shared=FAKE, C=1, rows=1,
            length=48, common=20, window=0, sinks=0, scale=1.0, status=FAKE, ws=None, ws_bytes=0):
    s = ctypes.byref(seq if seq is not None else _seq()) if seq is not False else None
    return lib.approxifer_attend_shared(s, Hq, Hkv, Dh, dtype, q, qs, kp, vp, out, groups, shared, C, rows, length, common, window, sinks, scale,
                                        status, ws, ws_bytes, None)


def test_attend_shared_refusals(lib):
    _sizes_are_refused(lib, _shared)
    assert _shared(lib, groups=None) == -1 and _shared(lib, shared=None) == -1
    assert _shared(lib, C=-1) == -2 and _shared(lib, common=-1) == -2 and _shared(lib, C=(1 << 20) + 1) == -3
    import torch
    need = binding.approxifer_attend_shared_workspace_bytes
    for args in ((0, 2, 1, 4, 2, 64), (4, 0, 1, 4, 2, 64), (4, 2, -1, 4, 2, 64), (4, 2, 1, 3, 2, 64), (4, 2, 1, 4, 2, 60)):
        assert need(*args, torch.float16, 1, 100, 50) == 0
    assert need(2, 2, 1, 4, 2, 64, torch.float16, 1, 100, -1) == 0
    assert need(2, 2, 1, 4, 2, 64, torch.float16, 1, 100, 50) % (2 * 4 * 66 * 4) == 0


def test_what_attend_shared_asks_for(lib):
    import torch
    need, plain = binding.approxifer_attend_shared_workspace_bytes, binding.approxifer_attend_workspace_bytes
    # shared: the sums, maximum and total of every row in two parts at least
    for T, B, C, heads, dtype, rows, length, common in ((24, 24, 1, (12, 12, 64), torch.float32, 1, 644, 500), (192, 192, 8, (32, 8, 128), torch.bfloat16, 1, 8500, 8000),
                                                        (40, 20, 2, (8, 4, 72), torch.float16, 2, 100, 50), (300, 300, 3, (8, 8, 256), torch.float32, 1, 600, 1)):
        each, got = T * heads[0] * (heads[2] + 2) * 4, need(T, B, C, *heads, dtype, rows, length, common)
        assert got >= 2 * each and got % each == 0, (T, B, C, heads, got)
    # not shared: what approxifer_attend() asks for
    for T, B, C, heads, dtype, rows, length, common in ((2, 2, 1, (4, 2, 64), torch.float16, 1, 100, 50), (16, 16, 8, (32, 8, 128), torch.bfloat16, 1, 9000, 8000),
                                                        (16 * 64, 16, 1, (32, 8, 128), torch.bfloat16, 64, 9000, 8000), (24, 24, 0, (12, 12, 64), torch.float32, 1, 9000, 8000),
                                                        (24, 24, 1, (12, 12, 64), torch.float32, 1, 9000, 0), (192, 24, 1, (24, 12, 64), torch.float32, 8, 9000, 8000)):
        assert need(T, B, C, *heads, dtype, rows, length, common) == plain(T, B, *heads, dtype, rows, length), (T, B, C, heads)
    assert plain(16, 16, 32, 8, 128, torch.bfloat16, 1, 9000) > 0
