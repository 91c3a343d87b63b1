"""Coded sequences whose cache runs out of room: nobody else notices, those that got none are told and no longer answer.

The same steps run on the GPU and, with the library's calls replaced by their references, on the CPU."""
import numpy as np
import pytest

G, K, N, S, PAGE, WIDTH, HEADS, KV, PROMPT = 3, 2, 4, 1, 4, 32, 4, 2, 9


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
    return torch.device("cpu")


def _served(device, pages, max_pages=20):
    import torch
    from paper_2109_09868_amd import sequences
    model = sequences.SequenceModel(2, WIDTH, HEADS, KV, 5, 3, device)
    cache = sequences.SequenceCache(2, HEADS, KV, WIDTH // HEADS, G * N, max_pages, pages, device, page=PAGE)
    cache.pools.fill_(7.0)
    served = sequences.CodedSequences(model, cache, G, K, N, S)
    served.start(torch.from_numpy(np.random.default_rng(5).standard_normal((PROMPT, WIDTH)).astype(np.float32)).to(device))
    return served


def _tokens(device, n, seed):
    import torch
    return torch.from_numpy(np.random.default_rng(seed).standard_normal((G, K, n, WIDTH)).astype(np.float32)).to(device)


def _arrival(device, seed, never=()):
    import torch
    t = np.random.default_rng(seed).exponential(1.0, (G, N)).astype(np.float32)
    for g, i in never:
        t[g, i] = np.inf
    return torch.from_numpy(t).to(device)


def _held(cache, b):
    """What sequence b holds, place by place: [layers, 2, KV, tokens, Dh]."""
    l = int(cache.lens[b])
    pages = cache.table[b, :-(-l // PAGE)].long()
    return cache.pools[:, :, pages].transpose(2, 3).flatten(3, 4)[:, :, :, :l].clone()


def test_pages_that_end_between_the_workers(device):
    # the prompt is two whole pages and a token in a third, of which every worker has a copy: 2 + 12 pages.  Four more tokens ask
    # for another page, and there are eight: those of the first two groups.  The last four places of the third group's sequences lie in a page
    # that all share.
    want, got = _served(device, 60), _served(device, 22)
    shared = [int(p) for p in got.cache.table[0, :2]]
    prompt = got.cache.pools[:, :, shared].clone()
    for n, seed in ((4, 11), (1, 12)):
        x, t = _tokens(device, n, seed), _arrival(device, seed)
        a, b = want.step(x, t), got.step(x, t)
        assert (a[1] == 0).all()
        assert (got.cache.pools[:, :, shared] == prompt).all()
        assert got.lost.tolist() == [[0] * N] * 2 + [[3] * N] and b[1].tolist() == [0, 0, 1]
        assert (a[0][:2] == b[0][:2]).all()
    for b in range(G * N):                                    # those that got no page keep what they had
        l = PROMPT + (5 if b < 2 * N else 0)
        assert int(got.cache.lens[b]) == l
        assert (_held(got.cache, b) == _held(want.cache, b)[:, :, :, :l]).all()
    # room or not, a sequence that has missed a token does not answer again, and takes no pages from the others
    x, t = _tokens(device, 2, 13), _arrival(device, 13)
    a, b = want.step(x, t), got.step(x, t)
    assert got.lost.tolist() == [[0] * N] * 2 + [[3] * N] and b[1].tolist() == [0, 0, 1] and (a[0][:2] == b[0][:2]).all()
    assert (got.cache.pools[:, :, shared] == prompt).all() and int(got.cache.lens[2 * N]) == PROMPT
    # not even if its group is all that goes on
    got.finish([2, 0])
    want.finish([2, 0])
    x, t = _tokens(device, 2, 14)[:2].contiguous(), _arrival(device, 14)[:2].contiguous()
    a, b = want.step(x, t), got.step(x, t)
    assert got.lost.tolist() == [[3] * N, [0] * N] and b[1].tolist() == [1, 0] and (a[0][1] == b[0][1]).all()


def test_workers_that_the_group_can_spare(device):
    # one worker of the last group gets no page: the others answer, as if it were late
    want, got = _served(device, 60), _served(device, 25)
    last = [(G - 1, N - 1)]
    for n, seed in ((3, 11), (1, 12), (2, 13), (1, 14)):
        x = _tokens(device, n, seed)
        a, b = want.step(x, _arrival(device, seed, last if n != 3 else ())), got.step(x, _arrival(device, seed))
        assert b[1].tolist() == [0] * G and (a[0] == b[0]).all()
    assert got.lost.tolist() == [[0] * N] * (G - 1) + [[0] * (N - 1) + [3]]


def test_tables_that_end(device):
    # three pages a sequence: the thirteenth token finds no place in the table, in none of them
    got = _served(device, 60, max_pages=3)
    got.step(_tokens(device, 3, 11), _arrival(device, 11))
    held = [_held(got.cache, b) for b in range(G * N)]
    _, status = got.step(_tokens(device, 1, 12), _arrival(device, 12))
    assert got.lost.tolist() == [[1] * N] * G and status.tolist() == [1] * G
    assert all((_held(got.cache, b) == held[b]).all() for b in range(G * N))


def test_a_prompt_that_is_not_copied_for_everybody(device):
    # 2 + 12 pages are needed, 12 are there: the last two forks are empty
    want, got = _served(device, 60), _served(device, 12)
    assert got.lost.tolist() == [[0] * N] * 2 + [[0, 0, 3, 3]]
    x = _tokens(device, 2, 11)
    a, b = want.step(x, _arrival(device, 11)), got.step(x, _arrival(device, 11))
    assert b[1].tolist() == [0, 0, 1] and (a[0][:2] == b[0][:2]).all()
    assert got.cache.lens.tolist() == [PROMPT + 2] * 10 + [0, 0]


def test_a_prompt_without_room(device):
    got = _served(device, 2)
    assert got.lost.tolist() == [[3] * N] * G
    _, status = got.step(_tokens(device, 1, 11), _arrival(device, 11))
    assert status.tolist() == [1] * G and not got.cache.lens.any() and (got.cache.pools == 7.0).all()


def test_a_cache_alone_tells_and_tries_again(device):
    # a shared page that is not full: refused, forked, then there is room
    import torch
    from paper_2109_09868_amd import sequences
    cache = sequences.SequenceCache(1, HEADS, KV, 8, 4, 4, 6, device, page=PAGE)
    cache.pools.fill_(7.0)
    cache.begin(1)
    assert cache.reserve(2).tolist() == [0]
    q = torch.from_numpy(np.random.default_rng(1).standard_normal((4, HEADS, 8)).astype(np.float32)).to(device)
    k = torch.from_numpy(np.random.default_rng(2).standard_normal((4, KV, 8)).astype(np.float32)).to(device)
    starts = torch.tensor([0, 2], dtype=torch.int32, device=device)
    cache.append(0, q[:2].contiguous(), k[:2], k[:2], starts)
    cache.refs[int(cache.table[0, 0])] += 1                   # a holder that is no sequence
    before = cache.pools.clone()
    assert cache.reserve(2).tolist() == [4] and cache.refused.tolist() == [4] and cache.lens.tolist() == [2]
    cache.append(0, q[2:].contiguous(), k[2:], k[2:], starts)
    assert (cache.attend(0, q[2:].contiguous(), starts, 2, 4) == 0).all() and (cache.pools == before).all()
    assert cache.fork([0]).tolist() == [0] and cache.reserve(2).tolist() == [0] and cache.lens.tolist() == [4]
    cache.append(0, q[2:].contiguous(), k[2:], k[2:], starts)
    out = cache.attend(0, q[2:].contiguous(), starts, 2, 4)
    assert not (out == 0).any() and (_held(cache, 0)[0, 1].transpose(0, 1) == k).all()
