"""approxifer_attend_shared against softmax and sums in 64 bits over every sequence's own pages."""
import math

import pytest
import torch

import sequence_reference as ref

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
ALL = list(ref.DTYPES.values())


@pytest.fixture(scope="module")
def binding():
    from paper_2109_09868_amd import binding
    binding.load()
    return binding


def _cache(seed, dtype, groups, shared, own, new, kv, dim, page, outside=()):
    """A cache whose group c has the sequences groups[c] .. groups[c + 1] - 1 with shared[c] places in common (as forks have them: full
    pages the same, the last one a copy) and own[b] of their own."""
    B = len(own)
    common = [0] * B
    for c, (x, y) in enumerate(zip(groups, groups[1:])):
        common[x:y] = [shared[c]] * (y - x)
    lens = [a + b for a, b in zip(common, own)]
    c = ref.cache(seed, dtype, lens, new, kv, dim, page)
    for x, y in zip(groups, groups[1:]):
        for b in range(x + 1, y):
            full, rest = divmod(common[b], page)
            c["table"][b, :full] = c["table"][x, :full]
            if rest:
                for pool in ("k_pool", "v_pool"):
                    c[pool][c["table"][b, full], :, :rest] = c[pool][c["table"][x, full], :, :rest]
    return c


def _i(x):
    return torch.tensor(x, dtype=torch.int32, device=DEV)


def _call(binding, c, q, groups, shared, window=0, sinks=0, scale=None, workspace=None, max_len=None, max_shared=None, q_device=None):
    kp, vp, table, lens, starts = ref.on(DEV, c)
    n = (c["starts"][1:] - c["starts"][:-1]).max()
    q = q.to(DEV) if q_device is None else q_device
    out = torch.full(q.shape, -3.0, dtype=q.dtype, device=DEV)
    status = torch.full((len(c["lens"]),), -1, dtype=torch.int32, device=DEV)
    binding.approxifer_attend_shared(q, kp, vp, table, lens, starts, _i(groups), _i(shared), int(n),
                                     int(c["lens"].max()) if max_len is None else max_len, max(shared) if max_shared is None else max_shared,
                                     window=window, sinks=sinks, scale=scale, out=out, status=status, workspace=workspace)
    return out.cpu(), status.tolist()


def _query(c, heads, dim, dtype, seed=7, big=1.0):
    return (big * torch.randn((c["T"], heads, dim), generator=torch.Generator().manual_seed(seed))).to(dtype)


def _apart(dtype, B, C, group, new):
    """Whether reading what is common for itself pays for what joining costs."""
    rows = group * new
    few = rows <= (12 * -(-rows // 16) if dtype == torch.float32 else 48)
    return few and B >= (3 if group > 1 else 2) * C


def _check(binding, dtype, groups, shared, own, new, heads, kv, dim, page, window=0, sinks=0, scale=None, big=1.0, apart=False):
    """apart: what is common has to be read for itself: the size of the workspace tells."""
    c = _cache(1, dtype, groups, shared, own, new, kv, dim, page)
    q = _query(c, heads, dim, dtype, big=big)
    want, bound = ref.attend(c, q, window, sinks, scale)
    B, n, longest = len(own), max(new), int(c["lens"].max())
    need = binding.approxifer_attend_shared_workspace_bytes(c["T"], B, len(shared), heads, kv, dim, dtype, n, longest, max(shared), window, sinks)
    each = 4 * c["T"] * heads * (dim + 2)
    assert not apart or (need > 0 and need % each == 0)
    spaces = [None, binding.NO_WORKSPACE]
    if need >= 2 * each:
        spaces.append(torch.full((2 * each,), 255, dtype=torch.uint8, device=DEV))         # NaN wherever it is not written
    for workspace in spaces:
        out, status = _call(binding, c, q, groups, shared, window, sinks, scale, workspace)
        assert status == [0] * B
        off = (out.double() - want).abs()
        assert torch.all(off <= bound), (float(off.max()), float((off / bound.clamp(min=1e-30)).max()))


HEADS = [(12, 12, 64, 16), (8, 2, 128, 16), (6, 3, 80, 8), (5, 1, 72, 32), (4, 4, 256, 64), (2, 1, 8, 1), (16, 1, 128, 16), (34, 2, 64, 16),
         (6, 2, 96, 128), (4, 2, 160, 256), (3, 3, 104, 16), (2, 2, 200, 16)]


@pytest.mark.parametrize("dtype", ALL, ids=list(ref.DTYPES))
@pytest.mark.parametrize("heads,kv,dim,page", HEADS)
def test_types_and_heads(binding, dtype, heads, kv, dim, page):
    _check(binding, dtype, [0, 5], [150], [1, 7, 64, 65, 20], [1] * 5, heads, kv, dim, page,
           apart=_apart(dtype, 5, 1, heads // kv, 1))                                                                    # tokens
    _check(binding, dtype, [0, 3, 7], [130, 67], [3, 7, 4, 33, 1, 2, 9], [1, 2, 1, 0, 1, 2, 1], heads, kv, dim, page)    # mixed
    _check(binding, dtype, [0, 3, 7], [130, 67], [3, 7, 4, 33, 1, 2, 9], [1] * 7, heads, kv, dim, page, window=40, sinks=3)


@pytest.mark.parametrize("dtype", ALL, ids=list(ref.DTYPES))
@pytest.mark.parametrize("kv,group", [(1, 1), (2, 4), (1, 8), (3, 3)])
@pytest.mark.parametrize("B,new", [(2, 1), (9, 1), (40, 1), (6, 5), (3, 16)])
def test_few_and_many_rows_of_a_group(binding, dtype, kv, group, B, new):
    own = [new + (7 * b) % 41 for b in range(B)]
    _check(binding, dtype, [0, B], [200], own, [new] * B, kv * group, kv, 64, 16, apart=_apart(dtype, B, 1, group, new))
    _check(binding, dtype, [0, B // 2, B], [33, 90], own, [new - b % 2 if new > 1 else 1 for b in range(B)], kv * group, kv, 128, 16)


@pytest.mark.parametrize("dtype", ALL, ids=list(ref.DTYPES))
@pytest.mark.parametrize("shared", [1, 15, 16, 17, 31, 32, 33, 63, 64, 65, 127, 128, 129, 255, 256, 257])
def test_lengths(binding, dtype, shared):
    _check(binding, dtype, [0, 3], [shared], [1, 2, 40], [1, 1, 1], 4, 2, 64, 16, apart=True)
    _check(binding, dtype, [0, 12], [shared], [1 + b for b in range(12)], [1] * 12, 8, 1, 128, 32, apart=True)
    _check(binding, dtype, [0, 3], [shared], [5, 6, 64], [5, 6, 2], 8, 1, 64, 4)


@pytest.mark.parametrize("dtype", ALL, ids=list(ref.DTYPES))
@pytest.mark.parametrize("window,sinks", [(1, 0), (1, 1), (2, 5), (31, 64), (64, 4), (65, 1), (90, 0), (90, 200), (300, 7), (1000, 3)])
def test_windows(binding, dtype, window, sinks):
    # windows that end before, inside and behind what is common; first tokens inside and behind it
    _check(binding, dtype, [0, 5], [150], [1, 7, 64, 110, 20], [1] * 5, 4, 2, 64, 16, window, sinks)
    _check(binding, dtype, [0, 20, 24], [133, 40], [1 + 9 * b % 97 for b in range(24)], [1] * 24, 8, 1, 128, 16, window, sinks)
    _check(binding, dtype, [0, 5], [150], [4, 7, 64, 110, 20], [4] * 5, 8, 1, 64, 8, window, sinks)


@pytest.mark.parametrize("dtype", ALL, ids=list(ref.DTYPES))
def test_long_sequences_are_split_and_joined(binding, dtype):
    _check(binding, dtype, [0, 3], [5000], [1, 1000, 2049], [1, 1, 1], 8, 2, 64, 16)
    _check(binding, dtype, [0, 2], [2100], [1, 2], [1, 1], 4, 4, 128, 64)
    _check(binding, dtype, [0, 24], [3000], [1 + b for b in range(24)], [1] * 24, 8, 1, 128, 16)
    _check(binding, dtype, [0, 2, 30], [300, 2500], [700] + [1 + b for b in range(29)], [1] * 30, 2, 1, 64, 16)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16], ids=["f32", "bf16"])
def test_large_scores(binding, dtype):
    for B in (3, 40):
        own = [1 + b for b in range(B)]
        _check(binding, dtype, [0, B], [300], own, [1] * B, 4, 2, 64, 16, big=40.0)
        _check(binding, dtype, [0, B], [300], own, [1] * B, 4, 2, 64, 16, scale=-2.0)
        _check(binding, dtype, [0, B], [300], own, [1] * B, 4, 2, 64, 16, scale=0.0)


@pytest.mark.parametrize("dtype", ALL, ids=list(ref.DTYPES))
@pytest.mark.parametrize("groups,shared", [([0, 0, 4, 4, 9], [5, 60, 7, 33]), ([2, 6], [50]), ([1, 1], [9]), ([3, 5, 7], [0, 70])])
def test_empty_groups_and_sequences_without_one(binding, dtype, groups, shared):
    _check(binding, dtype, groups, shared, [9 + b for b in range(9)], [1] * 9, 4, 2, 64, 16)
    _check(binding, dtype, groups, shared, [9 + b for b in range(9)], [b % 3 for b in range(9)], 8, 2, 64, 16)


@pytest.mark.parametrize("dtype", ALL, ids=list(ref.DTYPES))
def test_sequences_shorter_than_what_is_common(binding, dtype):
    # cut by a fork with `keep`: the rows lie inside what is common, and their sequences end there
    c = _cache(4, dtype, [0, 6], [100], [5, 1, 1, 30, 2, 1], [1] * 6, 2, 64, 16)
    for lens in ([37, 100, 64, 130, 1, 33], [37, 20, 64, 63, 1, 33]):
        c["lens"] = torch.tensor(lens, dtype=torch.int32)
        q = _query(c, 8, 64, dtype)
        for window, sinks in ((0, 0), (20, 3)):
            want, bound = ref.attend(c, q, window, sinks)
            out, status = _call(binding, c, q, [0, 6], [100], window, sinks)
            assert status == [0] * 6 and torch.all((out.double() - want).abs() <= bound)


@pytest.mark.parametrize("dtype", ALL, ids=list(ref.DTYPES))
@pytest.mark.parametrize("B", [3, 30])
def test_groups_that_cannot_be(binding, dtype, B):
    # a negative length, one beyond max_shared, sequences that there are not: all are attended to without sharing
    own = [40 + b for b in range(B)]
    c = _cache(6, dtype, [0, B], [60], own, [1] * B, 2, 64, 16)
    q = _query(c, 4, 64, dtype)
    want, bound = ref.attend(c, q)
    for groups, shared in (([0, B], [-1]), ([0, B], [61]), ([0, B], [2 ** 31 - 1]), ([0, B + 1], [60]), ([-1, B], [60]), ([-5, -3], [60]),
                           ([B + 3, B + 9], [60]), ([-2 ** 31, 2 ** 31 - 1], [60])):
        out, status = _call(binding, c, q, groups, shared, max_shared=60)
        assert status == [0] * B and torch.all((out.double() - want).abs() <= bound), (groups, shared)


@pytest.mark.parametrize("dtype", ALL, ids=list(ref.DTYPES))
@pytest.mark.parametrize("B", [4, 33])
def test_bad_sequences_do_not_disturb_the_others(binding, dtype, B):
    # the first, whose pages would be read, is too long; another has no place for its token; rows of a third lie outside
    own = [200] + [3 + b for b in range(1, B)]
    c = _cache(8, dtype, [0, B], [70], own, [1] * B, 2, 64, 16)
    q = _query(c, 8, 64, dtype)
    want, bound = ref.attend(c, q)
    c["lens"][2] = 0
    out, status = _call(binding, c, q, [0, B], [70], max_len=150)
    assert status == [1, 0, 0] + [0] * (B - 3)
    assert torch.all(out[0] == -3.0) and torch.all(out[2] == 0.0)
    ok = [1, *range(3, B)]
    assert torch.all((out[ok].double() - want[ok]).abs() <= bound[ok])
    c["starts"][B] = B + 5
    out, status = _call(binding, c, q, [0, B], [70], max_len=150)
    assert status == [1, 0, 0] + [0] * (B - 4) + [1]
    assert torch.all(out[B - 1] == -3.0) and torch.all((out[ok[:-1]].double() - want[ok[:-1]]).abs() <= bound[ok[:-1]])
    c["starts"][0] = -2
    out, status = _call(binding, c, q, [0, B], [70], max_len=290)
    assert status[0] == 1 and torch.all((out[ok[:-1]].double() - want[ok[:-1]]).abs() <= bound[ok[:-1]])


@pytest.mark.parametrize("dtype", ALL, ids=list(ref.DTYPES))
@pytest.mark.parametrize("B", [4, 33])
def test_bad_pages(binding, dtype, B):
    c = _cache(8, dtype, [0, B], [70], [3 + b for b in range(B)], [1] * B, 2, 64, 16)
    q = _query(c, 8, 64, dtype)
    want, bound = ref.attend(c, q, 20, 3)
    plain = ref.attend(c, q)
    c["table"][1, 4] = 9999                                   # only its own
    out, status = _call(binding, c, q, [0, B], [70])
    others = [0, *range(2, B)]
    assert status == [0, 2] + [0] * (B - 2)
    assert torch.all((out[others].double() - plain[0][others]).abs() <= plain[1][others])
    c["table"][0, 1] = -1                                     # of the one that is read for all
    out, status = _call(binding, c, q, [0, B], [70])
    assert status == [2] * B and torch.isnan(out).all()
    out, status = _call(binding, c, q, [0, B], [70], 20, 3)   # nobody's window reaches it
    far = [b for b in range(B) if int(c["lens"][b]) - 20 >= 32 and b != 1]
    assert all(status[b] == 0 for b in far) and torch.all((out[far].double() - want[far]).abs() <= bound[far])


@pytest.mark.parametrize("dtype", ALL, ids=list(ref.DTYPES))
@pytest.mark.parametrize("B", [3, 30])
@pytest.mark.parametrize("window,sinks", [(0, 0), (30, 3)])
def test_what_a_row_does_not_see_does_not_reach_it(binding, dtype, B, window, sinks):
    own = [2 + 3 * b % 37 for b in range(B)]
    c = _cache(5, dtype, [0, B], [90], own, [2] * B, 2, 64, 16)
    clean = {**c, "k_pool": c["k_pool"].clone(), "v_pool": c["v_pool"].clone()}
    q = _query(c, 8, 64, dtype)
    want, bound = ref.attend(clean, q, window, sinks)
    bad = {b: [int(c["lens"][b]) - 1] for b in range(0, B, 2)}                              # the first of two rows must not see it
    for b in range(B):
        bad.setdefault(b, [])
    if window:
        for j in range(sinks, 45):                            # before every window
            p = int(c["table"][0, j // 16])
            c["v_pool"][p, :, j % 16, j % 64], c["k_pool"][p, :, j % 16, (j + 3) % 64] = math.inf, math.nan
            for b in range(B):
                bad[b].append(j)
    for b in range(0, B, 2):
        p, s = int(c["table"][b, bad[b][0] // 16]), bad[b][0] % 16
        c["v_pool"][p, :, s, b % 64], c["k_pool"][p, :, s, (b + 5) % 64] = math.nan, -math.inf
    out, status = _call(binding, c, q, [0, B], [90], window, sinks)
    assert status == [0] * B
    checked = 0
    for b in range(B):
        for i in range(2):
            seen = ref.visible(int(c["lens"][b]) - 2 + i, int(c["lens"][b]), window, sinks)
            if not any(seen[j] for j in bad[b]):
                t = 2 * b + i
                assert torch.all((out[t].double() - want[t]).abs() <= bound[t]), (b, i)
                checked += 1
    assert checked >= B


@pytest.mark.parametrize("B", [3, 40])
def test_infinities_reach_the_rows_that_see_them(binding, B):
    c = _cache(5, torch.bfloat16, [0, B], [200], [1 + b for b in range(B)], [1] * B, 2, 64, 16)
    p = int(c["table"][0, 7])
    c["v_pool"][p, :, 3, 9] = math.inf
    q = _query(c, 8, 64, torch.bfloat16)
    out, status = _call(binding, c, q, [0, B], [200])
    assert status == [0] * B and torch.all(out[:, :, 9] == math.inf) and torch.isfinite(out[:, :, :9]).all() and torch.isfinite(out[:, :, 10:]).all()


@pytest.mark.parametrize("B,new,heads", [(5, 1, 4), (40, 1, 8), (6, 4, 8)])
def test_strides_graphs_and_streams(binding, B, new, heads):
    c = _cache(9, torch.bfloat16, [0, B], [333], [new + 5 * b for b in range(B)], [new] * B, 2, 128, 16)
    q = _query(c, heads, 128, torch.bfloat16)
    out, _ = _call(binding, c, q, [0, B], [333])
    wide = torch.empty((B * new, heads * 128 + 5), dtype=torch.bfloat16, device=DEV)
    for at in (0, 1):
        x = wide[:, at:at + heads * 128].unflatten(1, (heads, 128))
        x.copy_(q)
        assert torch.equal(_call(binding, c, q, [0, B], [333], q_device=x)[0], out)
    kp, vp, table, lens, starts = ref.on(DEV, c)
    longest, groups, shared = int(c["lens"].max()), _i([0, B]), _i([333])
    need = binding.approxifer_attend_shared_workspace_bytes(B * new, B, 1, heads, 2, 128, torch.bfloat16, new, longest, 333)
    ws = torch.empty((need,), dtype=torch.uint8, device=DEV)
    qd, o, st = q.to(DEV), torch.empty(q.shape, dtype=q.dtype, device=DEV), _i([-1] * B)
    side, graph = torch.cuda.Stream(), torch.cuda.CUDAGraph()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.graph(graph, stream=side):
        binding.approxifer_attend_shared(qd, kp, vp, table, lens, starts, groups, shared, new, longest, 333, out=o, status=st, workspace=ws)
    for _ in range(3):
        o.zero_()
        st.fill_(-1)
        ws.fill_(255)
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(o.cpu(), out) and st.tolist() == [0] * B
    # the graph reads lengths and tables when it runs: a token more in place of the last
    lens += 1
    table2 = c["table"].clone()
    o.zero_()
    torch.cuda.synchronize()
    got, _ = binding.approxifer_attend_shared(qd, kp, vp, table, lens - 1, starts, groups, shared, new, longest, 333, stream=side)
    side.synchronize()
    assert torch.equal(got.cpu(), out) and torch.equal(table.cpu(), table2)


def test_nothing_to_do_and_refusals(binding):
    c = _cache(2, torch.float16, [0, 2], [20], [3, 4], [0, 0], 2, 64, 16)
    kp, vp, table, lens, starts = ref.on(DEV, c)
    none = torch.empty((0, 4, 64), dtype=torch.float16, device=DEV)
    _, status = binding.approxifer_attend_shared(none, kp, vp, table, lens, starts, _i([0, 2]), _i([20]), 1, 24, 20)
    assert status.tolist() == [0, 0]
    q = torch.zeros((2, 4, 64), dtype=torch.float16, device=DEV)
    starts = _i([0, 1, 2])
    for groups, shared in ((_i([0]), _i([20])), (_i([0, 2]).long(), _i([20])), (_i([0, 2]), _i([20]).float()), (_i([0, 2]).cpu(), _i([20]))):
        with pytest.raises((TypeError, ValueError)):
            binding.approxifer_attend_shared(q, kp, vp, table, lens, starts, groups, shared, 1, 24, 20)
    with pytest.raises(binding.ApproxiferError) as e:
        binding.approxifer_attend_shared(q, kp, vp, table, lens, starts, _i([0, 2]), _i([20]), 1, 24, -1)
    assert e.value.code == -2
    out, status = binding.approxifer_attend_shared(q, kp, vp, table, lens, starts, _i([0]), _i([]), 1, 24, 20)
    assert status.tolist() == [0, 0] and torch.isfinite(out).all()


@pytest.mark.parametrize("dtype", ALL, ids=list(ref.DTYPES))
@pytest.mark.parametrize("heads,kv", [(2, 2), (8, 1), (48, 1)])
def test_more_groups_than_a_wave_has_lanes(binding, dtype, heads, kv):
    # 70 groups of one to four sequences, some of them empty; sequences of one to three new tokens
    sizes = [(3 * c) % 5 for c in range(70)]
    groups = [sum(sizes[:c]) for c in range(71)]
    B = groups[-1] + 3
    own = [3 + b % 5 for b in range(B)]
    assert B >= 2 * 70
    _check(binding, dtype, groups, [5 + (7 * c) % 40 for c in range(70)], own, [1] * B, heads, kv, 64, 16,
           apart=_apart(dtype, B, 70, heads // kv, 1))
    _check(binding, dtype, groups, [5 + (7 * c) % 40 for c in range(70)], own, [b % 3 for b in range(B)], 4, 2, 64, 16, window=20, sinks=2)


@pytest.mark.parametrize("dtype", ALL, ids=list(ref.DTYPES))
@pytest.mark.parametrize("heads,kv", [(5, 1), (33, 1)])
def test_more_groups_of_more_sequences(binding, dtype, heads, kv):
    sizes = [(3 * c) % 7 + 1 for c in range(70)]
    groups = [2 + sum(sizes[:c]) for c in range(71)]
    B = groups[-1] + 3
    assert _apart(dtype, B, 70, heads // kv, 1)
    _check(binding, dtype, groups, [5 + (7 * c) % 40 for c in range(70)], [3 + b % 5 for b in range(B)], [1] * B, heads, kv, 64, 16, apart=True)


@pytest.mark.parametrize("dtype", ALL, ids=list(ref.DTYPES))
@pytest.mark.parametrize("dim,page", [(8, 16), (64, 16), (64, 8), (40, 4), (160, 16), (192, 8), (200, 32), (256, 16), (256, 1)])
def test_rows_of_a_group_that_fill_tiles(binding, dtype, dim, page):
    # 272 rows, and 281 of sequences of one to three tokens of which a window takes some
    _check(binding, dtype, [0, 34], [150], [1 + b for b in range(34)], [1] * 34, 8, 1, dim, page, apart=True)
    new = [1 + b % 3 for b in range(36)]
    _check(binding, dtype, [1, 36], [150], [b + 3 for b in range(36)], new, 8, 2, dim, page, window=40, sinks=3, apart=True)


def test_a_first_group_behind_others_rows(binding):
    # groups that begin with the third sequence, whose rows are not the first
    _check(binding, torch.bfloat16, [2, 12, 40], [90, 300], [1 + b for b in range(43)], [1 + (b % 2) for b in range(43)], 16, 2, 128, 16, apart=True)
    _check(binding, torch.bfloat16, [35, 40], [300], [1 + b for b in range(43)], [1] * 43, 64, 2, 128, 16, apart=True)
