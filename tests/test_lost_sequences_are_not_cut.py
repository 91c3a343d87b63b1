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
