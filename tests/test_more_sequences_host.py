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
