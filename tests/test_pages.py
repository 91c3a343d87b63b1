"""The page operators against the same rules in plain Python: every index and every copied byte."""
import random

import pytest
import torch

import sequence_reference as ref

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


@pytest.fixture(scope="module")
def binding():
    from paper_2109_09868_amd import binding
    binding.load()
    return binding


def _state(rng, B, M, P, page, longest):
    """Sequences that hold pages at random places, some of them shared, some pages held by nobody we know."""
    refs, table, lens = [0] * P, [], []
    free = list(range(P))
    rng.shuffle(free)
    for b in range(B):
        row, l = [-1] * M, rng.randint(0, min(longest, M * page))
        if rng.random() < 0.3:
            l = l // page * page
        for j in range(-(-l // page)):
            if b and rng.random() < 0.2 and j < -(-lens[b - 1] // page) and (j + 1) * page <= min(l, lens[b - 1]):
                row[j] = table[b - 1][j]
            elif free:
                row[j] = free.pop()
            else:
                l = j * page
                break
            refs[row[j]] += 1
        table.append(row)
        lens.append(l)
    for p in rng.sample(range(P), P // 10):
        refs[p] += 1
    return table, lens, refs


def _i(x):
    return torch.tensor(x, dtype=torch.int32, device=DEV)


SIZES = [(1, 1, 1, 1, 1), (3, 4, 9, 2, 8), (5, 8, 60, 16, 100), (40, 6, 300, 8, 48), (70, 40, 5000, 16, 600), (1500, 3, 4000, 4, 12)]


@pytest.mark.parametrize("B,M,P,page,longest", SIZES)
@pytest.mark.parametrize("seed", range(3))
def test_reserve(binding, B, M, P, page, longest, seed):
    rng = random.Random(seed)
    table, lens, refs = _state(rng, B, M, P, page, longest)
    add = [rng.choice([0, 1, 1, rng.randint(0, 3 * page)]) for _ in range(B)]
    want = ref.reserve(table, lens, refs, add, page)
    t, l, r = _i(table), _i(lens), _i(refs)
    status = binding.approxifer_cache_reserve(t, l, r, _i(add), page)
    assert status.tolist() == want[3] and l.tolist() == want[1] and r.tolist() == want[2] and t.tolist() == want[0]


def test_reserve_until_the_pages_end(binding):
    # the third sequence finds too few, those behind it none; the fifth wants none
    t, l, r = _i([[-1] * 8 for _ in range(5)]), _i([0, 0, 0, 0, 3]), _i([0, 1, 0, 0, 0, 0, 1])
    t[4, 0] = 6
    status = binding.approxifer_cache_reserve(t, l, r, _i([8, 4, 12, 4, 1]), 4)
    assert status.tolist() == [0, 0, 3, 3, 0] and l.tolist() == [8, 4, 0, 0, 4]
    assert t[0, :2].tolist() == [0, 2] and t[1, 0] == 3 and t[2].tolist() == [-1] * 8 and r.tolist() == [1, 1, 1, 1, 0, 0, 1]


@pytest.mark.parametrize("P,each", [(40000, 9000), (30000, 9000), (9000, 9000), (20000, 3000)])
def test_reserve_more_than_one_list_of_pages(binding, P, each):
    rng = random.Random(P)
    refs = [int(rng.random() < 0.1) for _ in range(P)]
    table, lens, add = [[-1] * each for _ in range(4)], [0] * 4, [each] * 4
    want = ref.reserve(table, lens, refs, add, 1)
    t, l, r = _i(table), _i(lens), _i(refs)
    status = binding.approxifer_cache_reserve(t, l, r, _i(add), 1)
    assert status.tolist() == want[3] and l.tolist() == want[1] and r.tolist() == want[2] and t.tolist() == want[0]


def test_reserve_tells_what_is_wrong(binding):
    table = [[0, -1], [1, -1], [9, -1], [2, 3], [4, -1], [5, -1], [-1, -1]]
    lens, add = [3, 3, 3, 8, 3, -1, 0], [1, 2, 1, 1, -1, 1, 9]
    refs = [1, 2, 1, 1, 1, 1, 0, 0]
    want = ref.reserve(table, lens, refs, add, 4)
    assert want[3] == [0, 4, 2, 1, 1, 1, 1]
    t, l, r = _i(table), _i(lens), _i(refs)
    status = binding.approxifer_cache_reserve(t, l, r, _i(add), 4)
    assert status.tolist() == want[3] and l.tolist() == want[1] and r.tolist() == want[2] and t.tolist() == want[0]


def _pools(P, page, kv=2, dim=8, planes=3, dtype=torch.float16, seed=0):
    g = torch.Generator(device=DEV).manual_seed(seed)
    return torch.randn((planes, P, kv, page, dim), generator=g, device=DEV).to(dtype)


def _fork(binding, table, lens, refs, parents, keep, page, dtype=torch.float16, planes=3, dim=8):
    want = ref.fork(table, lens, refs, parents, keep, page)
    pools = _pools(len(refs), page, dim=dim, planes=planes, dtype=dtype)
    expect = pools.clone()
    for a, b in want[4]:
        expect[:, b] = pools[:, a]
    t, l, r = _i(table), _i(lens), _i(refs)
    got = binding.approxifer_cache_fork(pools, t, l, r, _i(parents), keep=_i(keep) if keep is not None else None)
    assert got[3].tolist() == want[3]
    assert got[1].tolist() == want[1] and got[0].tolist() == want[0] and got[2].tolist() == want[2]
    assert torch.equal(pools, expect)
    assert t.tolist() == table and l.tolist() == lens and r.tolist() == refs


@pytest.mark.parametrize("B,M,P,page,longest", SIZES)
@pytest.mark.parametrize("seed", range(3))
def test_fork(binding, B, M, P, page, longest, seed):
    rng = random.Random(seed)
    table, lens, refs = _state(rng, B, M, P, page, longest)
    n = rng.choice([1, B, 2 * B + 1])
    parents = [rng.randint(-1, B - 1) for _ in range(n)]
    keep = [rng.choice([M * page, rng.randint(0, longest)]) for _ in range(n)] if seed else None
    _fork(binding, table, lens, refs, parents, keep, page, dtype=(torch.float16, torch.float32, torch.bfloat16)[seed])


def test_fork_of_nothing_and_into_nothing(binding):
    _fork(binding, [[1, 0], [2, -1]], [3, 2], [1, 1, 1, 0], [-1, -1, -1], None, 2)
    _fork(binding, [[1, 0], [2, -1]], [3, 2], [1, 1, 1, 0], [1], None, 2)
    _fork(binding, [[1, 0], [2, -1]], [3, 2], [1, 1, 1, 0], [0, 0, 1, 0, 1, 1, 0], None, 2)   # the free pages end
    pools = _pools(4, 2)
    table, lens, refs, status = binding.approxifer_cache_fork(pools, _i([[1, 0], [2, -1]]), _i([3, 2]), _i([1, 1, 1, 0]), _i([]))
    assert table.shape == (0, 2) and refs.tolist() == [0, 0, 0, 0]


def test_fork_tells_what_is_wrong(binding):
    table, lens, refs = [[0, 1], [2, 9], [3, -1], [4, 5]], [4, 4, 99, 3], [1] * 6 + [0, 0]
    _fork(binding, table, lens, refs, [4, -2, 1, 2, 3, 0, 0, 3, 1], [9, 9, 9, 9, 9, -1, 3, 3, 2], 2)


def test_fork_shares_a_prompt(binding):
    # one prompt, 24 workers, in pages of several kilobytes and of one vector
    for page, dim, dtype in ((16, 128, torch.bfloat16), (1, 8, torch.float16), (64, 96, torch.float32)):
        l = 3 * page + page // 2
        n = -(-l // page)
        _fork(binding, [list(range(n)) + [-1]], [l], [1] * n + [0] * 40, [0] * 24, None, page, dtype=dtype, dim=dim, planes=4)


def test_fork_with_more_copies_than_a_list_holds(binding):
    n = 9001
    _fork(binding, [[0]], [1], [1] + [0] * (n - 50), [0] * n, None, 2, planes=1)


def _compact(binding, table, lens, refs, page, dtype=torch.float16):
    want = ref.compact(table, lens, refs, page)
    pools = _pools(len(refs), page, dtype=dtype)
    expect = pools.clone()
    for a, b in want[4]:
        expect[:, b] = pools[:, a]
    t, l, r = _i(table), _i(lens), _i(refs)
    moved, live = binding.approxifer_cache_compact(pools, t, l, r)
    assert live.tolist() == [want[3]] and moved.tolist() == want[2] and r.tolist() == want[1] and t.tolist() == want[0]
    assert torch.equal(pools, expect) and l.tolist() == lens


@pytest.mark.parametrize("B,M,P,page,longest", SIZES)
@pytest.mark.parametrize("seed", range(3))
def test_compact(binding, B, M, P, page, longest, seed):
    rng = random.Random(seed)
    table, lens, refs = _state(rng, B, M, P, page, longest)
    _compact(binding, table, lens, refs, page)


def test_compact_of_full_empty_and_reversed_pools(binding):
    _compact(binding, [[0, 1], [2, 3]], [4, 4], [1] * 4, 2)
    _compact(binding, [[-1, -1]], [0], [0] * 5, 2)
    for P in (2047, 2048, 2049):
        _compact(binding, [list(range(P - 1, P // 2, -1))], [P - 1 - P // 2], [0] * (P // 2 + 1) + [1] * (P - P // 2 - 1), 1)
    _compact(binding, [[7, 99, 0, -3]], [8], [0, 0, 0, 0, 0, 0, 0, 3], 2)        # entries that are no live page stay
    _compact(binding, [[3, 2], [7, 6]], [99, 4], [0, 0, 1, 1, 0, 0, 1, 1], 2)    # a length that cannot be


def test_the_page_calls_in_a_graph(binding):
    rng = random.Random(5)
    table, lens, refs = _state(rng, 9, 8, 100, 4, 30)
    parents = [rng.randint(-1, 8) for _ in range(12)]
    want = ref.fork(table, lens, refs, parents, None, 4)
    pools = _pools(100, 4)
    kept = pools.clone()
    t, l, r, p = _i(table), _i(lens), _i(refs), _i(parents)
    outs = [torch.empty((12, 8), dtype=torch.int32, device=DEV), _i([0] * 12), _i([0] * 100), _i([0] * 12)]
    ws = torch.empty((binding.approxifer_cache_workspace_bytes(9, 12, 100),), dtype=torch.uint8, device=DEV)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        binding.approxifer_cache_fork(pools, t, l, r, p, table_out=outs[0], lens_out=outs[1], refs_out=outs[2], status=outs[3],
                                      workspace=ws)
    for _ in range(4):
        pools.copy_(kept)
        ws.fill_(255)
        for o in outs:
            o.fill_(-5)
        graph.replay()
        torch.cuda.synchronize()
        assert [o.tolist() for o in outs] == [want[0], want[1], want[2], want[3]]
        for a, b in want[4]:
            assert torch.equal(pools[:, b], kept[:, a])
