"""Eviction of a cache whose pools hold nothing, or that has none: tables, lengths and masses are cut, nothing is copied."""
import pytest

import test_more_sequence_launches as more


def test_which_kernels_cut_without_pools(tmp_path, monkeypatch):
    # planes, heads and bytes of a row in the place of the two pools that the launches' program has
    old = 'at, 2, c["heads"][1], 256,'
    assert old in more._RUN
    monkeypatch.setattr(more, "_RUN", more._RUN.replace(old, "at if c['pools'][0] else None, *c['pools'],"))
    pools = [(0, 8, 16), (0, 8, 8), (0, 8, 0), (0, 0, 0), (0, 0, 256), (3, 0, 256), (3, 8, 0), (3, 8, 16)]
    calls = [dict(more.BASE, entry="evict", B=B, stride=5000, budget=100, pools=p) for p in pools for B in (1, 3, 5000)]
    for names in more._launches(tmp_path, calls):
        assert more._kinds(names) == ["evict_select", "evict_pages", "evict_move"]


@pytest.mark.gpu
@pytest.mark.parametrize("planes, heads, row_bytes", [(0, 4, 0), (0, 4, 8), (0, 0, 256), (2, 0, 256), (2, 4, 0)])
def test_cut_without_pools(planes, heads, row_bytes):
    import ctypes

    import torch
    from paper_2109_09868_amd import binding
    dev, page, budget = torch.device("cuda:0"), 16, 20
    lib, B, M, P = binding.load(), 3, 4, 16

    def ints(*shape, fill=None):
        return torch.tensor(fill, dtype=torch.int32, device=dev) if fill is not None else torch.full(shape, -7, dtype=torch.int32, device=dev)

    table = torch.arange(B * M, dtype=torch.int32, device=dev).view(B, M)
    lens, refs = ints(fill=[50, 20, 64]), ints(fill=[1] * (B * M) + [0] * (P - B * M))
    mass = torch.rand((B, 64), device=dev, generator=torch.Generator(dev).manual_seed(4))
    want = mass.cpu()
    kept, status = ints(B, budget), ints(B)
    need = binding.approxifer_cache_evict_workspace_bytes(B, budget, P, page)
    ws = torch.empty((need,), dtype=torch.uint8, device=dev)
    at = [ctypes.c_void_p(t.data_ptr()) for t in (table, lens, refs, mass, kept, status, ws)]
    torch.cuda.synchronize()
    assert lib.approxifer_cache_evict(*at[:4], 64, at[4], at[5], None, planes, heads, row_bytes, B, M, P, page, budget, 2, 5, at[6], need,
                                      None) == 0
    torch.cuda.synchronize()
    # 20 tokens are two pages; what the second one is not cut of it keeps, its table has four
    assert status.tolist() == [0, 0, 0] and lens.tolist() == [20, 20, 20]
    assert refs.tolist() == [1, 1, 0, 0] + [1, 1, 1, 1] + [1, 1, 0, 0] + [0] * 4
    assert table.tolist() == [[0, 1, -1, -1], [4, 5, 6, 7], [8, 9, -1, -1]]
    for b, n in ((0, 50), (2, 64)):
        inner = sorted(range(2, n - 5), key=lambda j: (-float(want[b, j]), j))[:budget - 7]
        places = [0, 1] + sorted(inner) + list(range(n - 5, n))
        assert kept[b].tolist() == places
        assert mass[b, :budget].tolist() == want[b, places].tolist() and not mass[b, budget:n].any()
    assert kept[1].tolist() == list(range(20)) and (mass[1].cpu() == want[1]).all()
