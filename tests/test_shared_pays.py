"""Where sequences that begin alike are attended to together: what the library says of it, and that a cache goes by it."""
import os

import pytest

from paper_2109_09868_amd import binding


@pytest.fixture(scope="module")
def lib():
    if not os.path.exists(binding.LIB_PATH):
        import __graft_entry__
        __graft_entry__.build()
    return binding.load()


def _pays(dtype, C, per, shared, own, Hq, Hkv, Dh, new=1, page=16, window=0, sinks=0):
    import torch
    t = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}[dtype]
    B = C * per
    return binding.approxifer_attend_shared_pays(B * new, B, C, Hq, Hkv, Dh, t, page, new, shared + own, shared, window, sinks)


def test_sizes_that_were_measured(lib):
    # microseconds of attend() and of the call that shares
    for taken, size in ((True, ("bf16", 1, 192, 8003, 512, 32, 8, 128)),              # 487, 120
                        (True, ("bf16", 9, 9, 1904, 24, 4, 4, 128)),                  # 40.8, 23.4
                        (True, ("f32", 1, 24, 500, 144, 12, 12, 64)),                 # 22.3, 18.2
                        (True, ("bf16", 32, 8, 512, 100, 8, 8, 128)),                 # 58.5, 51.5
                        (True, ("bf16", 1, 64, 2000, 100, 32, 8, 128, 8)),            # 70.4, 52.9
                        (False, ("bf16", 8, 8, 512, 100, 8, 8, 128)),                 # 18.5, 21.6
                        (False, ("bf16", 8, 4, 512, 100, 8, 8, 128)),                 # 11.6, 14.8
                        (False, ("f32", 1, 24, 100, 144, 12, 12, 64)),                # 12.5, 16.3
                        (False, ("f16", 8, 35, 336, 165, 32, 8, 96, 2)),              # 48.7, 79.8
                        (False, ("bf16", 1, 4, 4000, 100, 8, 8, 128)),                # 15.8, 17.2
                        (False, ("f16", 3, 27, 192, 87, 24, 12, 256))):               # 59.8, 70.6
        assert _pays(*size) is taken, size


def test_it_rises_with_what_is_common_and_falls_with_windows(lib):
    for dtype in ("f32", "f16", "bf16"):
        for heads in ((8, 8, 128), (12, 12, 64), (8, 1, 96)):
            got = [_pays(dtype, 2, 40, n, 200, *heads) for n in (1, 16, 100, 400, 1600, 6400, 25600)]
            assert got == sorted(got) and not got[0] and got[-1], (dtype, heads, got)
            for window in (1, 100, 200):                       # no window reaches what is common
                assert not _pays(dtype, 2, 40, 6400, 200, *heads, window=window)
            assert _pays(dtype, 2, 40, 25600, 200, *heads, window=25000)


def test_sizes_that_are_none(lib):
    import torch
    good = dict(T=192, B=192, C=1, Hq=32, Hkv=8, Dh=128, dtype=torch.bfloat16, page=16, max_rows=1, max_len=8500, max_shared=8000, window=0, sinks=0)
    assert binding.approxifer_attend_shared_pays(**good)
    for bad in (dict(T=0), dict(B=0), dict(C=0), dict(C=-1), dict(C=1 << 21), dict(Hq=33), dict(Hkv=0), dict(Dh=100), dict(Dh=264), dict(page=0),
                dict(page=12), dict(max_rows=0), dict(max_len=0), dict(max_shared=0), dict(max_shared=-1), dict(window=-1), dict(sinks=-1),
                dict(T=1 << 25), dict(C=192), dict(max_rows=100)):
        assert binding.approxifer_attend_shared_pays(**dict(good, **bad)) is False, bad


@pytest.mark.gpu
@pytest.mark.parametrize("length, window, taken", [(900, 0, True), (40, 0, False), (900, 64, False)])
def test_a_cache_reads_together_what_it_pays_to(monkeypatch, length, window, taken):
    import torch
    from paper_2109_09868_amd import sequences
    dev, heads, kv, dim, B = torch.device("cuda:0"), 8, 4, 64, 48
    cache = sequences.SequenceCache(1, heads, kv, dim, B, 60, 250, dev, window=window)
    calls = []
    for name in ("approxifer_attend", "approxifer_attend_shared"):
        f = getattr(binding, name)
        monkeypatch.setattr(binding, name, lambda *a, f=f, name=name, **k: (calls.append(name), f(*a, **k))[1])
    g = torch.Generator(dev).manual_seed(3)

    def draw(n, h):
        return torch.randn((n, h, dim), device=dev, generator=g)

    cache.begin(1)
    cache.reserve(length)
    k, v = draw(length + B, kv), draw(length + B, kv)
    cache.append(0, draw(length, heads), k[:length], v[:length], torch.tensor([0, length], dtype=torch.int32, device=dev))
    cache.fork([0] * B)
    cache.share([0, B], [length])
    cache.reserve(1)
    starts = torch.arange(B + 1, dtype=torch.int32, device=dev)
    q = cache.append(0, draw(B, heads), k[length:], v[length:], starts)
    assert not calls
    together = cache.attend(0, q, starts, 1, length + 1)
    assert calls == ["approxifer_attend_shared" if taken else "approxifer_attend"] and not cache.status.any()
    cache._common = None
    each = cache.attend(0, q, starts, 1, length + 1)
    # float32 on either side: a score is off by (64 + 8) 2^-24 |q| |k| / 8 at most (a rotation keeps lengths), twice that and the sums over the keys
    # in the result
    off = 2 * 2 * (72 * 2 ** -24 * float(q.norm(dim=-1).amax() * k.norm(dim=-1).amax()) / 8 + (length + 65) * 2 ** -24) * float(v.abs().amax())
    assert (together - each).abs().max() <= off and off < 0.1 and each.abs().max() > 0.1
