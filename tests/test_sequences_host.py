"""What the cached-sequence calls decide on the host, without a GPU: codes, refusals, sizes."""
import ctypes
import os
import re

import numpy as np
import pytest

from paper_2109_09868_amd import binding

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
FAKE = ctypes.c_void_p(4096)                                  # never dereferenced: every call below ends before a launch
ODD = ctypes.c_void_p(4097)


@pytest.fixture(scope="module")
def lib():
    if not os.path.exists(binding.LIB_PATH):
        import __graft_entry__
        __graft_entry__.build()
    return binding.load()


def _seq(T=4, B=2, M=3, P=5, page=16, table=4096, lens=4096, starts=4096):
    return binding._Sequences(table, lens, starts, T, B, M, P, page)


def _append(lib, seq=None, Hq=4, Hkv=2, Dh=64, dtype=0, q=FAKE, qs=256, k=FAKE, ks=128, v=FAKE, vs=128, out=FAKE, kp=FAKE, vp=FAKE,
            qw=None, kw=None, eps=1e-6, positions=None, axes=1, freq=(1.0,) * 32, axis=None, pairs=32, status=FAKE):
    f = (ctypes.c_double * max(len(freq), 1))(*freq) if freq is not None else None
    a = np.asarray(axis, np.int32).tobytes() if axis is not None else None
    s = ctypes.byref(seq if seq is not None else _seq()) if seq is not False else None
    return lib.approxifer_append(s, Hq, Hkv, Dh, dtype, q, qs, k, ks, v, vs, out, kp, vp, qw, kw, eps, positions, axes, f, a, pairs, 0,
                                 status, None)


def _attend(lib, seq=None, Hq=4, Hkv=2, Dh=64, dtype=0, q=FAKE, qs=256, kp=FAKE, vp=FAKE, out=FAKE, rows=1, length=48, window=0, sinks=0,
            scale=1.0, status=FAKE, ws=None, ws_bytes=0):
    s = ctypes.byref(seq if seq is not None else _seq()) if seq is not False else None
    return lib.approxifer_attend(s, Hq, Hkv, Dh, dtype, q, qs, kp, vp, out, rows, length, window, sinks, scale, status, ws, ws_bytes,
                                 None)


@pytest.mark.parametrize("call", [_append, _attend])
def test_sizes_of_caches_and_heads(lib, call):
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
    assert call(lib, _seq(B=0)) == -11                        # rows of no sequence
    assert call(lib, _seq(B=0, T=0, table=None, lens=None, starts=None)) == 0
    assert call(lib, _seq(T=0), status=None) == 0


def test_append_refusals(lib):
    for missing in ("q", "k", "v", "out", "kp", "vp"):
        assert _append(lib, **{missing: None}) == -1
    assert _append(lib, freq=None) == -1
    for bad in (dict(pairs=-1), dict(pairs=33), dict(axes=0), dict(axes=2), dict(eps=-1.0), dict(eps=float("nan")), dict(qs=255),
                dict(ks=127), dict(vs=0), dict(axis=[1] * 32), dict(axis=[-1] * 32), dict(axis=[0, 2] * 16, axes=2, positions=FAKE)):
        assert _append(lib, **bad) == -2, bad
    assert _append(lib, axes=5, positions=FAKE) == -3
    assert _append(lib, freq=[1.0] * 31 + [float("inf")]) == -4
    for odd in ("q", "k", "v", "out", "kp", "vp", "qw", "kw"):
        assert _append(lib, **{odd: ODD}) == -10, odd
    assert _append(lib, out=ctypes.c_void_p(4104)) == -10


def test_attend_refusals(lib):
    for missing in ("q", "kp", "vp", "out"):
        assert _attend(lib, **{missing: None}) == -1
    for bad in (dict(rows=-1), dict(length=-1), dict(window=-1), dict(sinks=-1), dict(scale=float("nan")), dict(scale=float("inf")),
                dict(qs=255)):
        assert _attend(lib, **bad) == -2, bad
    for odd in ("q", "kp", "vp", "out"):
        assert _attend(lib, **{odd: ODD}) == -10
    assert _attend(lib, ws=ODD, ws_bytes=1 << 20) == -10


def test_page_call_refusals(lib):
    r = lib.approxifer_cache_reserve
    for n, bad in enumerate([(-1, 3, 5, 16), (2, 0, 5, 16), (2, 3, 0, 16), (2, 3, 5, 12)]):
        assert r(FAKE, FAKE, FAKE, FAKE, None, *bad, None) == -11
    assert r(FAKE, FAKE, FAKE, FAKE, None, 2, 3, 5, 8192, None) == -3
    for n in range(4):
        assert r(*[None if n == m else FAKE for m in range(4)], None, 2, 3, 5, 16, None) == -1
    assert r(None, None, None, None, None, 0, 3, 5, 16, None) == 0

    def fork(args=(FAKE,) * 8 + (None,), pools=FAKE, planes=2, page_bytes=1024, sizes=(2, 3, 4, 5, 16), ws=FAKE, ws_bytes=1 << 20):
        return lib.approxifer_cache_fork(*args, pools, planes, page_bytes, *sizes, ws, ws_bytes, None)

    for n in (0, 1, 2, 3, 5, 6, 7):
        assert fork(tuple(None if n == m else FAKE for m in range(8)) + (None,)) == -1
    assert fork(pools=None) == -1 and fork(pools=ODD) == -10 and fork(page_bytes=1000) == -10 and fork(planes=-1) == -2
    assert fork(ws=None) == -12 and fork(ws_bytes=binding.approxifer_cache_workspace_bytes(2, 3, 5) - 1) == -12 and fork(ws=ODD) == -10
    assert fork(sizes=(2, -1, 4, 5, 16)) == -11 and fork(sizes=(2, 3, 4, 0, 16)) == -11 and fork(sizes=((1 << 20) + 1, 3, 4, 5, 16)) == -3

    def compact(args=(FAKE,) * 5, pools=FAKE, planes=2, page_bytes=1024, sizes=(2, 4, 5, 16), ws=FAKE, ws_bytes=1 << 20):
        return lib.approxifer_cache_compact(*args, pools, planes, page_bytes, *sizes, ws, ws_bytes, None)

    for n in range(5):
        assert compact(tuple(None if n == m else FAKE for m in range(5))) == -1
    assert compact(pools=None) == -1 and compact(pools=ODD) == -10 and compact(page_bytes=8) == -10 and compact(planes=-1) == -2
    assert compact(ws=None) == -12 and compact(ws_bytes=16) == -12 and compact(sizes=(2, 4, 0, 16)) == -11


def test_workspace_sizes(lib):
    assert binding.approxifer_cache_workspace_bytes(2, 3, 0) == 0 and binding.approxifer_cache_workspace_bytes(-1, 3, 5) == 0
    # room for every page's claim and every copy's two ends, for every second page's move
    for B, n, P in ((1, 1, 1), (100, 2400, 4096), (7, 0, 100000)):
        assert binding.approxifer_cache_workspace_bytes(B, n, P) >= 4 * max(P + 2 * n + 1, P + 1)
    import torch
    need = binding.approxifer_attend_workspace_bytes
    for args in ((0, 2, 4, 2, 64), (4, 0, 4, 2, 64), (4, 2, 3, 2, 64), (4, 2, 4, 2, 60), (4, 2, 4, 2, 264)):
        assert need(*args, torch.float16, 1, 100) == 0
    with pytest.raises(TypeError):
        need(4, 2, 4, 2, 64, torch.float64, 1, 100)


def test_rotary_frequencies(lib):
    f = binding.approxifer_rotary_frequencies(32, 500000.0)
    assert np.max(np.abs(f * 500000.0 ** (np.arange(32) / 32) - 1)) <= 1e-14 and f[0] == 1.0
    for bad in ((0, 1e4), (4, 0.0), (4, float("inf")), (4, -2.0)):
        with pytest.raises(binding.ApproxiferError) as e:
            binding.approxifer_rotary_frequencies(*bad)
        assert e.value.code == -2
    assert lib.approxifer_rotary_frequencies(4, 1e4, None) == -1


def test_pages_are_counted_in_31_bits(lib):
    # kernels walk over pages some thousands at a time, past the last one
    assert _attend(lib, _seq(P=(1 << 30) + 1)) == -3 and _append(lib, _seq(P=(1 << 30) + 1)) == -3
    assert lib.approxifer_cache_reserve(FAKE, FAKE, FAKE, FAKE, None, 2, 3, (1 << 30) + 1, 16, None) == -3
    assert binding.approxifer_cache_workspace_bytes(2, 3, (1 << 30) + 1) == 0 < binding.approxifer_cache_workspace_bytes(2, 3, 1 << 30)


def test_places_are_counted_in_31_bits(lib):
    # places are compared with those of a whole tile, or window, further on
    assert _attend(lib, _seq(M=(1 << 26) + 1)) == -3 and _attend(lib, _seq(M=(1 << 30) + 1, page=1)) == -3
    assert _append(lib, _seq(M=(1 << 30) + 1, page=1)) == -3


def test_bounds_beyond_any_sequence_ask_for_no_more(lib):
    import torch
    need = binding.approxifer_attend_workspace_bytes
    huge = 2 ** 63 - 1
    assert need(4, 2, 4, 2, 64, torch.float16, 1, huge) == need(4, 2, 4, 2, 64, torch.float16, 1, 1 << 30) > 0
    assert need(4, 2, 4, 2, 64, torch.float16, huge, huge, huge, huge) == need(4, 2, 4, 2, 64, torch.float16, 4, 1 << 30)
    assert need(400, 2, 4, 2, 64, torch.float32, 200, 9000, 500, huge) == need(400, 2, 4, 2, 64, torch.float32, 200, 9000, 500, 1 << 30)


def test_new_codes_have_texts_of_their_own(lib):
    texts = {binding.strerror(code) for code in range(0, -13, -1)}
    assert len(texts) == 13 and not any("unknown" in t for t in texts)


def test_constants_match_the_header():
    text = open(os.path.join(ROOT, "include", "approxifer.h")).read()
    c = dict(re.findall(r"#define\s+APPROXIFER_([A-Z0-9_]+)\s+\(?(-?\d+)\)?", text))
    assert (int(c["F32"]), int(c["F16"]), int(c["BF16"])) == (binding.F32, binding.F16, binding.BF16)
    for name in ("SEQUENCE_BAD", "SEQUENCE_BAD_PAGE", "SEQUENCE_NO_PAGES", "SEQUENCE_SHARED_PAGE"):
        assert int(c[name]) == getattr(binding, name)


def test_the_binding_refuses_what_is_no_device_tensor(lib):
    import torch
    x = torch.zeros((2, 4, 64))
    pool, table = torch.zeros((3, 2, 16, 64)), torch.zeros((1, 2), dtype=torch.int32)
    n = torch.zeros((2,), dtype=torch.int32)
    with pytest.raises(TypeError):
        binding.approxifer_attend(x, pool, pool, table, n[:1], n, 1, 8)
    with pytest.raises(TypeError):
        binding.approxifer_append(x, x[:, :2], x[:, :2], pool, pool, table, n[:1], n, np.ones(4))
    with pytest.raises(ValueError):
        binding.approxifer_append(x, x, x, pool, pool, table, n[:1], n, np.ones(4))
    with pytest.raises(TypeError):
        binding.approxifer_attend(x.double(), pool.double(), pool.double(), table, n[:1], n, 1, 8)
    with pytest.raises(TypeError):
        binding.approxifer_cache_reserve(table, n[:1], n, n[:1], 16)
    with pytest.raises(TypeError):
        binding.approxifer_cache_fork(pool, table, n[:1], torch.zeros((3,), dtype=torch.int32), n)
    with pytest.raises(TypeError):
        binding.approxifer_cache_compact(pool, table, n[:1], torch.zeros((3,), dtype=torch.int32))


def test_scales_that_float32_does_not_hold(lib):
    # the kernels multiply by scale log2(e) in float32
    for scale in (1e300, -1e300, 3.4e38, -2.0 ** 127):
        assert _attend(lib, scale=scale) == -2, scale
    for scale in (2.0 ** 126, -2.0 ** 126, 1e-300, 0.0):
        assert _attend(lib, _seq(B=0, T=0), scale=scale) == 0, scale
