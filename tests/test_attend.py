"""approxifer_attend against softmax and sums in 64 bits."""
import math

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


def _call(binding, c, q, window=0, sinks=0, scale=None, workspace=None, max_rows=None, max_len=None, q_device=None):
    kp, vp, table, lens, starts = ref.on(DEV, c)
    n = (c["starts"][1:] - c["starts"][:-1]).max()
    q = q.to(DEV) if q_device is None else q_device
    out = torch.full(q.shape, -3.0, dtype=q.dtype, device=DEV)
    status = torch.full((len(c["lens"]),), -1, dtype=torch.int32, device=DEV)
    binding.approxifer_attend(q, kp, vp, table, lens, starts, int(n) if max_rows is None else max_rows,
                              int(c["lens"].max()) if max_len is None else max_len, window=window, sinks=sinks, scale=scale, out=out,
                              status=status, workspace=workspace)
    return out.cpu(), status.tolist()


def _check(binding, dtype, lens, new, heads, kv, dim, page, window=0, sinks=0, scale=None, seed=0, big=1.0, layouts=False):
    c = ref.cache(seed, dtype, lens, new, kv, dim, page)
    q = (big * torch.randn((c["T"], heads, dim), generator=torch.Generator().manual_seed(seed + 50))).to(dtype)
    want, bound = ref.attend(c, q, window, sinks, scale)
    for workspace in (None, binding.NO_WORKSPACE):
        out, status = _call(binding, c, q, window, sinks, scale, workspace)
        assert status == [0] * len(lens)
        off = (out.double() - want).abs()
        assert torch.all(off <= bound), (float(off.max()), float((off / bound.clamp(min=1e-30)).max()))
    if layouts:
        wide = torch.empty((c["T"], heads * dim + 5), dtype=dtype, device=DEV)
        for at in (0, 1):
            x = wide[:, at:at + heads * dim].unflatten(1, (heads, dim))
            x.copy_(q)
            got, _ = _call(binding, c, q, window, sinks, scale, q_device=x)
            assert torch.equal(got, _call(binding, c, q, window, sinks, scale)[0])


@pytest.mark.parametrize("dtype", list(ref.DTYPES.values()), ids=list(ref.DTYPES))
@pytest.mark.parametrize("heads,kv,dim,page", [(12, 12, 64, 16), (8, 2, 128, 16), (6, 3, 80, 8), (5, 1, 72, 32), (4, 4, 256, 64),
                                               (2, 1, 8, 1), (16, 1, 128, 16), (34, 2, 64, 16), (6, 2, 96, 128), (4, 2, 160, 256),
                                               (3, 3, 104, 16), (2, 2, 200, 16)])
def test_types_and_heads(binding, dtype, heads, kv, dim, page):
    _check(binding, dtype, [1, 7, 40, 33, 129], [1, 2, 40, 0, 1], heads, kv, dim, page, layouts=True)        # mixed
    _check(binding, dtype, [1, 7, 64, 65, 200], [1, 1, 1, 1, 1], heads, kv, dim, page)                        # tokens
    _check(binding, dtype, [1, 7, 64, 65, 200], [1, 1, 1, 1, 1], heads, kv, dim, page, window=30, sinks=3)
    _check(binding, dtype, [150, 97], [150, 97], heads, kv, dim, page, window=33, sinks=2)                    # prompts


@pytest.mark.parametrize("dtype", list(ref.DTYPES.values()), ids=list(ref.DTYPES))
@pytest.mark.parametrize("window,sinks", [(0, 0), (1, 0), (1, 1), (2, 5), (16, 0), (31, 64), (64, 4), (65, 1), (300, 7), (1000, 3)])
def test_windows(binding, dtype, window, sinks):
    _check(binding, dtype, [257, 64, 3], [257, 10, 3], 4, 2, 64, 16, window, sinks)
    _check(binding, dtype, [257, 64, 3], [1, 1, 1], 4, 2, 64, 16, window, sinks)


@pytest.mark.parametrize("dtype", list(ref.DTYPES.values()), ids=list(ref.DTYPES))
@pytest.mark.parametrize("length", [1, 2, 15, 16, 17, 31, 32, 33, 63, 64, 65, 127, 128, 129, 255, 256, 257])
def test_lengths(binding, dtype, length):
    _check(binding, dtype, [length], [1], 8, 1, 128, 16)
    _check(binding, dtype, [length], [length], 2, 1, 64, 32)
    _check(binding, dtype, [length + 100], [length], 2, 2, 128, 16)


@pytest.mark.parametrize("dtype", list(ref.DTYPES.values()), ids=list(ref.DTYPES))
def test_long_sequences_are_split_and_joined(binding, dtype):
    _check(binding, dtype, [5000, 1, 2049], [1, 1, 1], 8, 2, 64, 16)
    _check(binding, dtype, [4100], [1], 4, 4, 128, 64)
    _check(binding, dtype, [3000, 2000], [3, 2], 4, 2, 128, 16)
    _check(binding, dtype, [3000], [40], 4, 2, 64, 16)
    _check(binding, dtype, [5000, 300], [1, 1], 8, 2, 64, 16, window=2000, sinks=100)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16], ids=["f32", "bf16"])
def test_large_scores(binding, dtype):
    # scores of hundreds: only differences from the running maximum are exponentiated
    _check(binding, dtype, [300, 80], [1, 80], 4, 2, 64, 16, big=40.0)
    _check(binding, dtype, [300, 80], [1, 80], 4, 2, 64, 16, scale=-2.0)
    _check(binding, dtype, [90], [90], 4, 2, 64, 16, scale=0.0)


@pytest.mark.parametrize("dtype", list(ref.DTYPES.values()), ids=list(ref.DTYPES))
@pytest.mark.parametrize("new", [1, 5, 70])
@pytest.mark.parametrize("window,sinks", [(0, 0), (20, 3)])
def test_what_a_row_does_not_see_does_not_reach_it(binding, dtype, new, window, sinks):
    # values and keys that are no numbers at every seventh place: the rows that see none of them stay exact
    lens = [200, 131]
    c = ref.cache(5, dtype, lens, [new, new], 2, 64, 16)
    clean = {**c, "k_pool": c["k_pool"].clone(), "v_pool": c["v_pool"].clone()}
    poison = {0: math.nan, 1: math.inf, 2: -math.inf}
    bad = [[], []]
    for b in range(2):
        for n, j in enumerate(range(lens[b] - new // 2 - 1, lens[b] - 40 if new == 1 else lens[b], 1)):
            bad[b].append(j)
        if window:
            bad[b] += list(range(sinks, lens[b] - new - window - 3))
        for n, j in enumerate(bad[b]):
            p, s = int(c["table"][b, j // 16]), j % 16
            c["v_pool"][p, :, s, n % 64] = poison[n % 3]
            c["k_pool"][p, :, s, (n + 5) % 64] = poison[(n + 1) % 3]
    q = torch.randn((2 * new, 4, 64), generator=torch.Generator().manual_seed(1)).to(dtype)
    want, bound = ref.attend(clean, q, window, sinks)
    out, status = _call(binding, c, q, window, sinks)
    checked = 0
    for b in range(2):
        for i in range(new):
            seen = ref.visible(lens[b] - new + i, lens[b], window, sinks)
            if not any(seen[j] for j in bad[b]):
                t = b * new + i
                assert torch.all((out[t].double() - want[t]).abs() <= bound[t]), (b, i)
                checked += 1
    assert checked > 0 and status == [0, 0]


@pytest.mark.parametrize("dtype", list(ref.DTYPES.values()), ids=list(ref.DTYPES))
@pytest.mark.parametrize("new", [1, 70])
def test_what_a_row_sees_does_reach_it(binding, dtype, new):
    c = ref.cache(6, dtype, [150], [new], 1, 64, 16)
    for j, x in ((20, math.inf), (21, math.nan), (22, -math.inf)):
        c["v_pool"][int(c["table"][0, j // 16]), 0, j % 16, j] = x
    q = torch.randn((new, 2, 64), generator=torch.Generator().manual_seed(1)).to(dtype)
    out, _ = _call(binding, c, q)
    assert torch.all(out[:, :, 20] == math.inf) and torch.all(out[:, :, 21].isnan()) and torch.all(out[:, :, 22] == -math.inf)
    rest = [d for d in range(64) if d not in (20, 21, 22)]
    assert torch.all(out[:, :, rest].isfinite())


@pytest.mark.parametrize("dtype", list(ref.DTYPES.values()), ids=list(ref.DTYPES))
@pytest.mark.parametrize("length", [1, 33, 150])
def test_the_last_value_of_a_row_may_be_infinite(binding, dtype, length):
    # lengths that end inside a tile: places behind the last take nothing of it
    c = ref.cache(6, dtype, [length], [1], 1, 64, 16)
    j = length - 1
    c["v_pool"][int(c["table"][0, j // 16]), 0, j % 16, 9] = math.inf
    q = torch.randn((1, 2, 64), generator=torch.Generator().manual_seed(1)).to(dtype)
    out, _ = _call(binding, c, q)
    assert torch.all(out[:, :, 9] == math.inf) and int(out.isfinite().sum()) == 2 * 63


@pytest.mark.parametrize("new", [1, 40])
def test_many_small_weights_of_half_precision_count(binding, new):
    # 6000 keys of a weight that is next to 2^-26 of the first one's: half precision has no numbers there.  Weights are kept as
    # 2^7 times themselves, so that each is off by 2^-32 of the largest at most, and by half a step.
    c = ref.cache(0, torch.float16, [6000], [new], 1, 64, 16)
    c["k_pool"].zero_()
    p = int(c["table"][0, 0])
    c["k_pool"][p, 0, 0, 0] = 4.5
    c["v_pool"][:] = 1.0
    c["v_pool"][p, 0, 0] = 0.0
    q = torch.zeros((new, 4, 64), dtype=torch.float16)
    q[:, :, 0] = 4.0
    out, _ = _call(binding, c, q, scale=1.0)
    n = torch.arange(6000 - new, 6000, dtype=torch.float64)
    small = math.exp(-18.0)
    want = n * small / (1 + n * small)
    bound = n * 2.0 ** -32 + want * (2 * ref.half_step(torch.float16) + (6000 + 64 + 36 * 64) * ref.U32)
    assert torch.all((out.double() - want[:, None, None]).abs() <= bound[:, None, None])


@pytest.mark.parametrize("status", [True, False])
def test_bounds_of_zero(binding, status):
    c = ref.cache(0, torch.float16, [40, 7000], [1, 1], 2, 64, 16)
    kp, vp, table, lens, starts = ref.on(DEV, c)
    lib, q, out = binding.load(), torch.zeros((2, 4, 64), dtype=torch.float16, device=DEV), torch.full((2, 4, 64), -3.0, device=DEV).half()
    st, ws = torch.full((2,), -1, dtype=torch.int32, device=DEV), torch.empty((1 << 22,), dtype=torch.uint8, device=DEV)
    for T, rows in ((2, 0), (0, 0), (0, 1)):
        seq = binding._Sequences(table.data_ptr(), lens.data_ptr(), starts.data_ptr(), T, 2, table.shape[1], kp.shape[0], 16)
        rc = lib.approxifer_attend(seq, 4, 2, 64, binding.F16, q.data_ptr(), 256, kp.data_ptr(), vp.data_ptr(), out.data_ptr(), rows, 7000,
                                   0, 0, 0.125, st.data_ptr() if status else None, ws.data_ptr(), ws.numel(), None)
        assert rc == 0
    torch.cuda.synchronize()
    assert torch.all(out == -3.0) and st.tolist() == ([1, 1] if status else [-1, -1])


def test_what_a_call_on_a_stream_allocates_belongs_to_it(binding):
    c = ref.cache(0, torch.bfloat16, [7000], [1], 2, 64, 16)
    kp, vp, table, lens, starts = ref.on(DEV, c)
    q = torch.randn((1, 8, 64), generator=torch.Generator().manual_seed(1)).to(torch.bfloat16)
    want, _ = _call(binding, c, q)
    x, side = q.to(DEV), torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    for stream in (side, side.cuda_stream):
        out, status = binding.approxifer_attend(x, kp, vp, table, lens, starts, 1, 7000, stream=stream)
        side.synchronize()
        assert status.tolist() == [0] and torch.equal(out.cpu(), want)


@pytest.mark.parametrize("dtype", list(ref.DTYPES.values()), ids=list(ref.DTYPES))
@pytest.mark.parametrize("new", [3, 70])
def test_rows_that_see_nothing_are_zero(binding, dtype, new):
    # more new tokens than the sequence has: the first rows have no place
    c = ref.cache(7, dtype, [2, 0, 66], [new, new, new], 2, 64, 16)
    q = torch.randn((3 * new, 4, 64), generator=torch.Generator().manual_seed(1)).to(dtype)
    want, bound = ref.attend(c, q)
    out, status = _call(binding, c, q)
    assert status == [0, 0, 0]
    assert torch.all((out.double() - want).abs() <= bound)
    assert torch.all(out[:new - 2] == 0) and torch.all(out[new:2 * new] == 0)


@pytest.mark.parametrize("dtype", list(ref.DTYPES.values()), ids=list(ref.DTYPES))
@pytest.mark.parametrize("new", [1, 3, 90])
def test_bad_sequences_and_pages(binding, dtype, new):
    lens = [100, 100, 100, 100, 100]
    c = ref.cache(8, dtype, lens, [new] * 5, 2, 64, 16)
    P = c["k_pool"].shape[0]
    c["table"][1, 1] = P
    c["table"][2, 5] = -1
    c["lens"][3] = 16 * 7 + 1
    q = torch.randn((5 * new, 4, 64), generator=torch.Generator().manual_seed(1)).to(dtype)
    good = {**c, "table": c["table"].clamp(0, P - 1), "lens": torch.tensor([100, 100, 100, 0, 100], dtype=torch.int32)}
    want, bound = ref.attend(good, q)
    out, status = _call(binding, c, q, max_len=100)
    assert status == [0, 2, 2, 1, 0]
    for b in range(5):
        for i in range(new):
            t, place = b * new + i, 100 - new + i
            if b == 3:
                assert torch.all(out[t] == -3.0)
            elif (b == 1 and place >= 16) or (b == 2 and place >= 80):
                assert torch.all(out[t].isnan()), (b, i)
            else:
                assert torch.all((out[t].double() - want[t]).abs() <= bound[t]), (b, i)
    # a window hides the bad page: nobody sees it, nobody is told; a window of 10 from place 99 ends in page 5, one of 4 does not
    if new == 1:
        _, status = _call(binding, c, q, window=10, max_len=100)
        assert status == [0, 0, 2, 1, 0]
        _, status = _call(binding, c, q, window=4, max_len=100)
        assert status == [0, 0, 0, 1, 0]
    # bounds that a sequence does not keep
    _, status = _call(binding, c, q, max_len=99)
    assert status == [1] * 5
    if new > 1:
        out, status = _call(binding, c, q, max_rows=new - 1, max_len=100)
        assert status == [1] * 5 and torch.all(out == -3.0)
    # rows that are not there
    c["starts"] = torch.tensor([0, new, 2 * new, 9 * new, 4 * new, 5 * new], dtype=torch.int32)
    _, status = _call(binding, c, q, max_rows=new, max_len=100)
    assert status[0] == 0 and status[2:4] == [1, 1]


def test_offsets_beyond_32_bits(binding):
    # a pool of more than 2^32 bytes and 2^31 values: the sequence's pages lie at its very end
    P, kv, page, dim = 270000, 4, 16, 128
    k = torch.empty((P, kv, page, dim), dtype=torch.float16, device=DEV)
    v = torch.empty((P, kv, page, dim), dtype=torch.float16, device=DEV)
    assert k.numel() > 2 ** 31
    c = ref.cache(9, torch.float16, [100, 33], [1, 33], kv, dim, page)
    used = c["k_pool"].shape[0]
    k[P - used:], v[P - used:] = c["k_pool"].to(DEV), c["v_pool"].to(DEV)
    q = torch.randn((34, 8, dim), generator=torch.Generator().manual_seed(1)).half()
    want, bound = ref.attend(c, q)
    for max_rows, rows in ((33, slice(0, 34)), (1, slice(0, 1))):
        starts = c["starts"] if max_rows == 33 else torch.tensor([0, 1, 1], dtype=torch.int32)
        out, _ = binding.approxifer_attend(q[rows].to(DEV), k, v, (c["table"] + (P - used)).to(DEV), c["lens"].to(DEV), starts.to(DEV),
                                           max_rows, 100)
        assert torch.all((out.cpu().double() - want[rows]).abs() <= bound[rows])
    del k, v
    torch.cuda.empty_cache()


def test_no_rows(binding):
    c = ref.cache(0, torch.float32, [5, 0], [0, 0], 2, 64, 16)
    out, status = _call(binding, c, torch.empty((0, 4, 64)), max_rows=1)
    assert out.shape == (0, 4, 64) and status == [0, 0]


@pytest.mark.parametrize("lens,new", [([700, 80], [1, 1]), ([300, 170], [300, 70])])
def test_same_bits_every_time_on_any_stream_and_in_graphs(binding, lens, new):
    c = ref.cache(0, torch.bfloat16, lens, new, 2, 64, 16)
    q = torch.randn((c["T"], 8, 64), generator=torch.Generator().manual_seed(1)).to(torch.bfloat16)
    first, _ = _call(binding, c, q)
    kp, vp, table, lens_, starts = ref.on(DEV, c)
    x, out, status = q.to(DEV), torch.empty(q.shape, dtype=q.dtype, device=DEV), torch.empty((2,), dtype=torch.int32, device=DEV)
    need = binding.approxifer_attend_workspace_bytes(c["T"], 2, 8, 2, 64, q.dtype, max(new), max(lens))
    workspace = torch.empty((max(need, 1),), dtype=torch.uint8, device=DEV)

    def call():
        binding.approxifer_attend(x, kp, vp, table, lens_, starts, max(new), max(lens), out=out, status=status, workspace=workspace)

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        out.fill_(9.0)
        call()
    side.synchronize()
    assert torch.equal(out.cpu(), first)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        call()
    for _ in range(4):
        out.fill_(7.0)
        workspace.fill_(255)
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out.cpu(), first) and status.tolist() == [0, 0]


@pytest.mark.parametrize("dtype", list(ref.DTYPES.values()), ids=list(ref.DTYPES))
@pytest.mark.parametrize("length,new", [(300, 1), (300, 70), (300, 300), (9000, 70)])
@pytest.mark.parametrize("gap", [12.0, 30.0, 80.0])
def test_an_infinity_of_a_small_weight_reaches_the_rows_that_see_it(binding, dtype, length, new, gap):
    # every key's score is 0 but that of one at place 20, which is `gap` below: in half precision its weight rounds to 0, and 0 times an
    # infinity would be no number
    c = ref.cache(6, dtype, [length], [new], 1, 64, 16)
    c["k_pool"].zero_()
    p = int(c["table"][0, 1])
    c["k_pool"][p, 0, 4, 0] = -gap / 4
    q = torch.zeros((new, 2, 64), dtype=dtype)
    q[:, :, 0] = 4.0
    want, bound = ref.attend(c, q, scale=1.0)
    c["v_pool"][p, 0, 4, 5], c["v_pool"][p, 0, 4, 6] = math.inf, -math.inf
    out, status = _call(binding, c, q, scale=1.0)
    sees = torch.arange(length - new, length) >= 20
    assert status == [0]
    assert torch.all(out[sees][:, :, 5] == math.inf) and torch.all(out[sees][:, :, 6] == -math.inf)
    off, rest = (out.double() - want).abs(), [d for d in range(64) if d not in (5, 6)]
    assert torch.all(off[~sees] <= bound[~sees]) and torch.all(off[:, :, rest] <= bound[:, :, rest])
