"""approxifer_cache_evict against the same rules in plain Python: every index, every mass and every byte of the pools."""
import math
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


def _i(x):
    return torch.tensor(x, dtype=torch.int32, device=DEV)


def _state(rng, B, M, P, page, lengths, shared):
    """Sequences at random pages; a share of their full pages are the sequence's before them."""
    refs, table, lens = [0] * P, [], []
    free = list(range(P))
    rng.shuffle(free)
    for b in range(B):
        l, row = rng.choice(lengths) if isinstance(lengths, list) else rng.randint(0, lengths), [-1] * M
        for j in range(-(-l // page)):
            if b and rng.random() < shared and (j + 1) * page <= min(l, lens[b - 1]):
                row[j] = table[b - 1][j]
            else:
                row[j] = free.pop()
            refs[row[j]] += 1
        table.append(row)
        lens.append(l)
    return table, lens, refs


def _masses(rng, B, L, ties=False):
    draw = (lambda: float(rng.choice([0.0, 0.25, 1.0]))) if ties else (lambda: 0.0 if rng.random() < 0.1 else math.exp(rng.gauss(0, 2)))
    return torch.tensor([[draw() for _ in range(L)] for _ in range(B)], dtype=torch.float32).tolist()


def _check(binding, table, lens, refs, mass, budget, first, recent, page, planes=3, kv=2, dim=8, dtype=torch.float16, **given):
    want = ref.evict(table, lens, refs, mass, budget, first, recent, page)
    P = len(refs)
    g = torch.Generator(device=DEV).manual_seed(3)
    pools = torch.randn((planes, P, kv, page, dim), generator=g, device=DEV).to(dtype)
    expect = pools.clone()
    if want[6]:
        (sp, ss), (tp, ts) = (torch.tensor([m[n] for m in want[6]], device=DEV).t() for n in (0, 1))
        expect[:, tp, :, ts] = pools[:, sp, :, ss]
    t, l, r, m = _i(table), _i(lens), _i(refs), torch.tensor(mass, dtype=torch.float32, device=DEV)
    kept, status = binding.approxifer_cache_evict(pools, t, l, r, m, budget, first, recent, **given)
    assert status.tolist() == want[5]
    assert kept.tolist() == want[4] and l.tolist() == want[1] and t.tolist() == want[0] and r.tolist() == want[2]
    assert torch.equal(m, torch.tensor(want[3], dtype=torch.float32, device=DEV)) or any(math.isnan(x) for row in mass for x in row)
    assert torch.equal(pools, expect)
    return want


@pytest.mark.parametrize("dtype,kv,dim", [(torch.float32, 3, 64), (torch.float16, 2, 8), (torch.bfloat16, 1, 128), (torch.float16, 5, 80),
                                          (torch.float32, 1, 256), (torch.bfloat16, 2, 200)])
@pytest.mark.parametrize("page", [1, 4, 16])
def test_types_and_heads(binding, dtype, kv, dim, page):
    rng = random.Random(dim + page)
    table, lens, refs = _state(rng, 6, -(-90 // page) + 1, 700, page, 90, 0.3)
    mass = _masses(rng, 6, 95)
    for budget, first, recent in ((1, 0, 0), (1, 1, 0), (1, 0, 1), (17, 2, 5), (40, 0, 0), (40, 40, 0), (40, 0, 40), (200, 3, 3)):
        _check(binding, table, lens, refs, mass, budget, first, recent, page, 3, kv, dim, dtype)


@pytest.mark.parametrize("shared", [0.0, 0.5, 1.0])
@pytest.mark.parametrize("ties", [False, True])
@pytest.mark.parametrize("seed", range(4))
def test_sequences_with_and_without_shared_pages(binding, shared, ties, seed):
    rng = random.Random(seed)
    B, page = rng.choice([1, 5, 40]), rng.choice([2, 8, 16])
    table, lens, refs = _state(rng, B, 300 // page + 2, 12000 // page, page, [0, 1, 30, 63, 64, 65, 200, 300], shared)
    for p in rng.sample(range(len(refs)), 5):                 # holders that are no sequence
        refs[p] += 1
    mass = _masses(rng, B, 300, ties)
    for budget, first, recent in ((64, 0, 0), (64, 4, 16), (63, 0, 8), (65, 1, 0), (250, 4, 100)):
        _check(binding, table, lens, refs, mass, budget, first, recent, page)


@pytest.mark.parametrize("length,budget", [(4097, 4096), (5000, 2500), (9001, 100), (20000, 12289), (70000, 33333)])
def test_long_sequences(binding, length, budget):
    rng = random.Random(length)
    table, lens, refs = _state(rng, 2, length // 16 + 1, length // 4, 16, [length], 0.1)
    _check(binding, table, lens, refs, _masses(rng, 2, length), budget, 4, budget // 5, 16, planes=2, kv=1)
    _check(binding, table, lens, refs, _masses(rng, 2, length, True), budget, 0, 0, 16, planes=1, kv=1)


def test_masses_that_are_no_ordinary_numbers(binding):
    inf, nan = math.inf, math.nan
    mass = [[nan, 1.0, inf, -inf, -0.0, 0.0, -2.5, 1e-45, nan, 3e38, inf, -1e-45, 2.0, nan, -3e38, 0.0]]
    table, refs = [[3, 1, 0, 2]], [1, 1, 1, 1, 0]
    for budget in range(1, 16):
        want = ref.evict(table, [16], refs, mass, budget, 0, 0, 4)
        m, l, t, r = torch.tensor(mass, device=DEV), _i([16]), _i(table), _i(refs)
        kept, status = binding.approxifer_cache_evict(torch.zeros((1, 5, 1, 4, 8), device=DEV), t, l, r, m, budget)
        assert kept.tolist() == want[4] and status.tolist() == [0]
        assert torch.equal(m.cpu().nan_to_num(nan=7.0), torch.tensor(want[3]).nan_to_num(nan=7.0))
    # all the same: the first of them stay
    kept, _ = binding.approxifer_cache_evict(torch.zeros((1, 5, 1, 4, 8), device=DEV), _i(table), _i([16]), _i(refs),
                                             torch.full((1, 16), nan, device=DEV), 6, recent=2)
    assert kept.tolist() == [[0, 1, 2, 3, 14, 15]]


def test_pages_that_run_out_and_a_last_page_that_others_hold(binding):
    # all three share the two first pages; one page is free: the first sequence takes it, the others stay as they are
    table, refs = [[0, 1, 2, -1], [0, 1, 3, -1], [0, 1, 4, -1]], [3, 3, 1, 1, 1, 0, 7]
    mass = [[1.0] * 4 + [0.0] + [1.0] * 7] * 3
    want = _check(binding, table, [12] * 3, refs, mass, 8, 0, 0, 4)
    assert want[5] == [0, 3, 3] and want[1] == [8, 12, 12] and want[2] == [3, 2, 0, 1, 1, 1, 7]
    # nothing moves, but the last page is shared and no longer full
    want = _check(binding, table, [12] * 3, refs, [[9.0] * 6 + [0.0] * 6] * 3, 6, 0, 0, 4)
    assert want[5] == [0, 3, 3] and want[0][0] == [0, 5, -1, -1]
    want = _check(binding, table, [12] * 3, refs, [[9.0] * 8 + [0.0] * 4] * 3, 8, 0, 0, 4)
    assert want[5] == [0, 0, 0] and want[0] == [[0, 1, -1, -1]] * 3


def test_what_is_wrong_with_a_sequence_is_told_and_leaves_it_alone(binding):
    table = [[0, 1], [2, 99], [3, -1], [4, 5], [6, 7], [8, 9], [10, 11]]
    refs = [1] * 11 + [0] * 3
    lens, mass = [8, 8, 7, 9, -1, 4, 8], [[float(j) for j in range(8)]] * 7
    want = _check(binding, table, lens, refs, mass, 4, 1, 1, 4)
    assert want[5] == [0, 2, 2, 1, 1, 0, 2]                   # the last one's second page has no holder
    want = _check(binding, table, lens, refs, [row[:7] for row in mass], 4, 1, 1, 4)
    assert want[5] == [1, 1, 2, 1, 1, 0, 1]                   # longer than its masses


def test_without_pools_sequences_or_statuses(binding):
    table, lens, refs, mass = [[0, 1], [2, 3]], [8, 6], [1] * 4, [[float(-j) for j in range(8)]] * 2
    want = ref.evict(table, lens, refs, mass, 5, 1, 1, 4)
    t, l, r, m = _i(table), _i(lens), _i(refs), torch.tensor(mass, device=DEV)
    kept = _i([[0] * 5] * 2)
    ws = torch.empty((binding.approxifer_cache_evict_workspace_bytes(2, 5, 4, 4),), dtype=torch.uint8, device=DEV)
    rc = binding.load().approxifer_cache_evict(t.data_ptr(), l.data_ptr(), r.data_ptr(), m.data_ptr(), 8, kept.data_ptr(), None, None, 0, 2,
                                               16, 2, 2, 4, 4, 5, 1, 1, ws.data_ptr(), ws.numel(), None)
    torch.cuda.synchronize()
    assert rc == 0 and kept.tolist() == want[4] and t.tolist() == want[0] and r.tolist() == want[2] and m.tolist() == want[3]
    none = torch.empty((0, 2), dtype=torch.int32, device=DEV)
    kept, status = binding.approxifer_cache_evict(torch.zeros((1, 4, 1, 4, 8), device=DEV), none, none[:, 0], r,
                                                  torch.empty((0, 8), device=DEV), 5)
    assert kept.shape == (0, 5) and status.shape == (0,)


def test_in_a_graph_on_another_stream_and_twice_in_a_row(binding):
    rng = random.Random(8)
    table, lens, refs = _state(rng, 7, 20, 200, 8, [100, 150, 33], 0.4)
    mass = _masses(rng, 7, 160)
    want = ref.evict(table, lens, refs, mass, 60, 2, 9, 8)
    once = ref.evict(want[0], want[1], want[2], want[3], 31, 0, 5, 8)
    pools = torch.randn((2, 200, 2, 8, 16), device=DEV)
    expect = pools.clone()
    for moves in (want[6], once[6]):
        now = expect.clone()
        for (sp, ss), (tp, ts) in moves:
            expect[:, tp, :, ts] = now[:, sp, :, ss]
    before = [_i(table), _i(lens), _i(refs), torch.tensor(mass, device=DEV), pools.clone()]
    t, l, r, m = (x.clone() for x in before[:4])
    kept = [torch.empty((7, n), dtype=torch.int32, device=DEV) for n in (60, 31)]
    status = _i([-1] * 7)
    ws = torch.empty((binding.approxifer_cache_evict_workspace_bytes(7, 60, 200, 8),), dtype=torch.uint8, device=DEV)
    side, graph = torch.cuda.Stream(), torch.cuda.CUDAGraph()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.graph(graph, stream=side):
        binding.approxifer_cache_evict(pools, t, l, r, m, 60, 2, 9, kept=kept[0], status=status, workspace=ws)
        binding.approxifer_cache_evict(pools, t, l, r, m, 31, 0, 5, kept=kept[1], status=status, workspace=ws)
    for _ in range(4):
        for x, y in zip((t, l, r, m, pools), before):
            x.copy_(y)
        ws.fill_(255)
        graph.replay()
        torch.cuda.synchronize()
        assert [t.tolist(), l.tolist(), r.tolist()] == [list(x) for x in once[:3]] and m.tolist() == once[3]
        assert kept[0].tolist() == want[4] and kept[1].tolist() == once[4] and torch.equal(pools, expect)
    for x, y in zip((t, l, r, m, pools), before):
        x.copy_(y)
    torch.cuda.synchronize()
    kept, status = binding.approxifer_cache_evict(pools, t, l, r, m, 60, 2, 9, stream=side)
    side.synchronize()
    assert kept.tolist() == want[4] and status.tolist() == want[5] and t.tolist() == want[0]


def test_refusals_of_the_binding(binding):
    t, l, r, m = _i([[0, 1]]), _i([8]), _i([1, 1]), torch.zeros((1, 8), device=DEV)
    pools = torch.zeros((2, 2, 1, 4, 8), device=DEV)
    ws = torch.empty((1 << 16,), dtype=torch.uint8, device=DEV)
    for args in (dict(mass=m[0]), dict(mass=m.half()), dict(mass=m.cpu()), dict(lens=l.long()), dict(refs=_i([1, 1, 0])),
                 dict(pools=pools[:, :, :, :, :4]), dict(kept=_i([[0] * 3])), dict(status=_i([0, 0])), dict(workspace=ws.cpu())):
        call = dict(dict(pools=pools, table=t, lens=l, refs=r, mass=m, budget=4, workspace=ws), **args)
        with pytest.raises((TypeError, ValueError)):
            binding.approxifer_cache_evict(**call)
    for args, code in ((dict(budget=0), -2), (dict(first=5), -2), (dict(recent=-1), -2), (dict(first=3, recent=2), -2),
                       (dict(workspace=ws[:16]), -12), (dict(workspace=binding.NO_WORKSPACE), -12), (dict(workspace=ws[1:]), -10)):
        call = dict(dict(pools=pools, table=t, lens=l, refs=r, mass=m, budget=4, workspace=ws), **args)
        with pytest.raises(binding.ApproxiferError) as e:
            binding.approxifer_cache_evict(**call)
        assert e.value.code == code, args
    assert l.tolist() == [8] and t.tolist() == [[0, 1]]
