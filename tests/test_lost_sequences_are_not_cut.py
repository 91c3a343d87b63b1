"""Coded sequences that are cut while workers are lost: the lost ones are left alone, take no pages from the others, and keep what was first
told of them.

The same steps run on the GPU and, with the library's calls replaced by their references, on the CPU."""
import numpy as np
import pytest

K, N, S, PAGE, WIDTH, HEADS, KV, PROMPT = 2, 4, 1, 4, 32, 4, 2, 38


def _attend_mass(q, k_pool, v_pool, table, lens, starts, mass, max_rows, max_len, window=0, sinks=0, out=None, status=None, workspace=None):
    import sequence_reference as ref
    c = {"k_pool": k_pool, "v_pool": v_pool, "table": table, "lens": lens, "starts": starts, "page": k_pool.shape[2]}
    for b, m in enumerate(ref.mass(c, q, window, sinks)[0]):
        mass[b, :len(m)] += m.to(mass.dtype)
    out.copy_(ref.attend(c, q, window, sinks)[0])
    status.zero_()


def _evict(pools, table, lens, refs, mass, budget, first=0, recent=0, kept=None, status=None, workspace=None):
    import torch
    import sequence_reference as ref
    got = ref.evict(table.tolist(), lens.tolist(), refs.tolist(), mass.tolist(), budget, first, recent, pools.shape[-2])
    before = pools.clone()
    for t, values in zip((table, lens, refs, mass, kept, status), got):
        t.copy_(torch.tensor(values).reshape(t.shape))
    for (p, i), (r, j) in got[6]:
        pools[:, :, r, :, j] = before[:, :, p, :, i]


@pytest.fixture(params=["references", pytest.param("library", marks=pytest.mark.gpu)])
def device(request, monkeypatch):
    import torch
    from paper_2109_09868_amd import binding
    if request.param == "library":
        return torch.device("cuda:0")
    import cpu_sequences
    if binding._lib is None:
        import os
        if not os.path.exists(binding.LIB_PATH):
            import __graft_entry__
            __graft_entry__.build()
    cpu_sequences.replace(monkeypatch, binding)
    monkeypatch.setattr(binding, "approxifer_attend_mass", _attend_mass)
    monkeypatch.setattr(binding, "approxifer_cache_evict", _evict)
    return torch.device("cpu")


def _served(device, pages):
    """One group behind a prompt of ten pages, the last of them copied for three of its four workers; a cut to 24 tokens moves all that is
    behind a sequence's first token: six pages for each."""
    import torch
    from paper_2109_09868_amd import sequences
    model = sequences.SequenceModel(2, WIDTH, HEADS, KV, 5, 3, device)
    cache = sequences.SequenceCache(2, HEADS, KV, WIDTH // HEADS, N, 12, pages, device, page=PAGE, weigh=True)
    served = sequences.CodedSequences(model, cache, 1, K, N, S)
    served.start(torch.from_numpy(np.random.default_rng(5).standard_normal((PROMPT, WIDTH)).astype(np.float32)).to(device))
    cache.mass.fill_(1.0)
    cache.mass[:, 0] = 0.0
    return served


def _told(cache, b, status):
    """Sequence b is lost, as append() and attend() tell it."""
    cache.status.zero_()
    cache.status[b] = status
    cache.lose()
    cache._settle()


def _answer(served, device, seed):
    import torch
    x = np.random.default_rng(seed).standard_normal((1, K, 1, WIDTH)).astype(np.float32)
    return served.step(torch.from_numpy(x).to(device), torch.arange(1.0, N + 1.0, device=device).view(1, N))


def test_a_second_status_does_not_change_the_first(device):
    # eviction tells of refused sequences too, as append() and attend() do not
    served = _served(device, 10 + 3 + 6)
    cache = served.cache
    _told(cache, 0, 2)
    for told in ([2, 0, 3, 3], [2, 0, 3, 3], [3, 0, 1, 0]):
        cache.status.copy_(cache.status.new_tensor(told))
        cache.lose()
        assert served.lost.tolist() == [[2, 0, 3, 3]] and cache.whole.tolist() == [False, True, False, False]
    for expected in (24, 23):
        served.evict(expected)
        assert served.lost.tolist()[0][0] == 2 and max(served.lost.tolist()[0]) == 3


def test_a_lost_worker_takes_no_pages(device):
    served = _served(device, 10 + 3 + 18)
    cache = served.cache
    _told(cache, 0, 2)
    before, masses, table = cache.lens.tolist(), cache.mass[0].clone(), cache.table[0].clone()
    kept = served.evict(24)
    assert cache.status.tolist() == [0, 0, 0, 0] and served.lost.tolist() == [[2, 0, 0, 0]]
    assert cache.lens.tolist() == [before[0], 24, 24, 24] and (cache.table[0] == table).all() and (cache.mass[0] == masses).all()
    assert (kept[0] == -1).all() and kept[1:].tolist() == [list(range(1, 25))] * 3
    _, status = _answer(served, device, 6)
    assert status.tolist() == [0] and served.lost.tolist() == [[2, 0, 0, 0]] and cache.lens.tolist() == [before[0], 25, 25, 25]


def test_what_was_told_first_stays(device):
    served = _served(device, 10 + 3 + 6)
    cache = served.cache
    _told(cache, 0, 2)
    cache.table[0, 3] = -1                                    # as its status says: a page of it is none
    served.evict(24)
    assert served.lost.tolist() == [[2, 0, 3, 3]] and cache.lens.tolist() == [PROMPT, 24, PROMPT, PROMPT]
    for budget in (23, 8):                                    # the cut sequence alone, again
        served.evict(budget)
        assert served.lost.tolist() == [[2, 0, 3, 3]] and cache.lens.tolist() == [PROMPT, budget, PROMPT, PROMPT]
    # statuses of a call that does not pass over them
    cache.status.copy_(cache.refused)
    cache.lose()
    assert served.lost.tolist() == [[2, 0, 3, 3]] and cache.whole.tolist() == [False, True, False, False]


def test_a_refused_sequence_is_cut_and_has_room_again(device):
    from paper_2109_09868_amd import sequences
    cache = sequences.SequenceCache(1, HEADS, KV, 8, 2, 4, 5, device, page=PAGE, weigh=True)
    cache.begin(2)
    assert cache.reserve(8).tolist() == [0, 0] and cache.reserve(8).tolist() == [3, 3]
    cache.evict(4, 1, 1)
    assert cache.status.tolist() == [0, 0] and cache.lens.tolist() == [4, 4] and cache.refused.tolist() == [3, 3]
    assert cache.reserve(4).tolist() == [0, 0] and cache.lens.tolist() == [8, 8]
    # one of them, as reserve() has it
    assert cache.reserve(8).tolist() == [3, 3]
    lost = cache.refused.clone()
    lost[1] = 0
    kept = cache.evict(4, 1, 1, lost=lost)
    assert cache.lens.tolist() == [8, 4] and cache.refused.tolist() == [3, 0] and (kept[0] == -1).all() and (kept[1] >= 0).all()
    assert cache.whole.tolist() == [False, True] and cache.dropped.tolist() == [4, 8]


def test_positions_are_looked_up_once_a_step(device, monkeypatch):
    import torch
    served = _served(device, 10 + 3 + 24)
    cache, asked, f = served.cache, [], torch.searchsorted
    monkeypatch.setattr(torch, "searchsorted", lambda *a, **k: (asked.append(a[1].numel()), f(*a, **k))[1])
    _answer(served, device, 6)
    assert asked == []                                        # nothing has been cut: positions are places
    served.evict(24)
    _answer(served, device, 7)
    assert asked == [N] and served.lost.tolist() == [[0] * N]
    # two tokens of one, none of another: behind the 40 that each has had
    starts = torch.tensor([0, 2, 2, 3, 4], dtype=torch.int32, device=device)
    cache.reserve(torch.tensor([2, 0, 1, 1], dtype=torch.int32, device=device))
    assert cache.positions(4, starts).tolist() == [40, 41, 40, 40]
