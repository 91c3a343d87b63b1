"""approxifer_attend_mass against softmax and its sums in 64 bits."""
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


def _least(binding, T, heads):
    return torch.empty((-(-8 * T * heads // 256) * 256,), dtype=torch.uint8, device=DEV)


def _call(binding, c, q, before, window=0, sinks=0, scale=None, workspace=None, max_rows=None, max_len=None):
    kp, vp, table, lens, starts = ref.on(DEV, c)
    n = (c["starts"][1:] - c["starts"][:-1]).max()
    out = torch.full(q.shape, -3.0, dtype=q.dtype, device=DEV)
    status = torch.full((len(c["lens"]),), -1, dtype=torch.int32, device=DEV)
    mass = before.to(DEV)
    binding.approxifer_attend_mass(q.to(DEV), kp, vp, table, lens, starts, mass, int(n) if max_rows is None else max_rows,
                                   int(c["lens"].max()) if max_len is None else max_len, window=window, sinks=sinks, scale=scale, out=out,
                                   status=status, workspace=workspace)
    return out.cpu(), mass.cpu(), status.tolist()


def _check(binding, dtype, lens, new, heads, kv, dim, page, window=0, sinks=0, scale=None, seed=0, big=1.0, behind=5):
    c = ref.cache(seed, dtype, lens, new, kv, dim, page)
    g = torch.Generator().manual_seed(seed + 50)
    q = (big * torch.randn((c["T"], heads, dim), generator=g)).to(dtype)
    want, bound = ref.attend(c, q, window, sinks, scale)
    sums, off = ref.mass(c, q, window, sinks, scale)
    before = torch.rand((len(lens), max(lens) + behind), generator=g) * 3.0
    total = before.double()
    total[:, :max(lens)] += sums
    allowed = torch.zeros_like(total)
    allowed[:, :max(lens)] = off + ref.U32 * torch.where(sums > 0, total[:, :max(lens)], 0.0)
    for workspace in (None, _least(binding, c["T"], heads)):
        out, mass, status = _call(binding, c, q, before, window, sinks, scale, workspace)
        assert status == [0] * len(lens)
        assert torch.all((out.double() - want).abs() <= bound)
        far = (mass.double() - total).abs()
        assert torch.all(far <= allowed), (float(far.max()), float((far / allowed.clamp(min=1e-30)).max()))


@pytest.mark.parametrize("dtype", ALL, ids=list(ref.DTYPES))
@pytest.mark.parametrize("heads,kv,dim,page", [(12, 12, 64, 16), (8, 2, 128, 16), (6, 3, 80, 8), (5, 1, 72, 32), (4, 4, 256, 64),
                                               (2, 1, 8, 1), (16, 1, 128, 16), (34, 2, 64, 16), (6, 2, 96, 128), (4, 2, 160, 256),
                                               (3, 3, 104, 16), (2, 2, 200, 16)])
def test_types_and_heads(binding, dtype, heads, kv, dim, page):
    _check(binding, dtype, [1, 7, 40, 33, 129], [1, 2, 40, 0, 1], heads, kv, dim, page)                       # mixed
    _check(binding, dtype, [1, 7, 64, 65, 300], [1, 1, 1, 1, 1], heads, kv, dim, page)                        # tokens
    _check(binding, dtype, [1, 7, 64, 65, 200], [1, 1, 1, 1, 1], heads, kv, dim, page, window=30, sinks=3)
    _check(binding, dtype, [150, 97], [150, 97], heads, kv, dim, page, window=33, sinks=2)                    # prompts


@pytest.mark.parametrize("dtype", ALL, ids=list(ref.DTYPES))
@pytest.mark.parametrize("window,sinks", [(0, 0), (1, 0), (1, 1), (2, 5), (31, 64), (64, 4), (65, 1), (300, 7), (1000, 3)])
def test_windows(binding, dtype, window, sinks):
    _check(binding, dtype, [330, 64, 3], [330, 10, 3], 4, 2, 64, 16, window, sinks)
    _check(binding, dtype, [600, 64, 3], [1, 1, 1], 4, 2, 64, 16, window, sinks)
    _check(binding, dtype, [600, 64, 3], [70, 3, 1], 4, 1, 128, 16, window, sinks)


@pytest.mark.parametrize("dtype", ALL, ids=list(ref.DTYPES))
@pytest.mark.parametrize("length", [1, 2, 15, 16, 17, 31, 32, 33, 63, 64, 65, 127, 128, 129, 255, 256, 257])
def test_lengths(binding, dtype, length):
    _check(binding, dtype, [length], [1], 8, 1, 128, 16, behind=0)
    _check(binding, dtype, [length], [length], 2, 1, 64, 32, behind=0)
    _check(binding, dtype, [length + 100], [length], 2, 2, 128, 16)


@pytest.mark.parametrize("dtype", ALL, ids=list(ref.DTYPES))
def test_long_sequences(binding, dtype):
    _check(binding, dtype, [5000, 1, 2049], [1, 1, 1], 8, 2, 64, 16)
    _check(binding, dtype, [4100], [1], 4, 4, 128, 64)
    _check(binding, dtype, [3000, 2000], [3, 2], 4, 2, 128, 16)
    _check(binding, dtype, [3000], [40], 4, 2, 64, 16)
    _check(binding, dtype, [5000, 300], [1, 1], 8, 2, 64, 16, window=2000, sinks=100)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16], ids=["f32", "bf16"])
def test_large_scores(binding, dtype):
    _check(binding, dtype, [300, 80], [1, 80], 4, 2, 64, 16, big=40.0)
    _check(binding, dtype, [300, 80], [1, 80], 4, 2, 64, 16, scale=-2.0)
    _check(binding, dtype, [90, 90], [90, 1], 4, 2, 64, 16, scale=0.0)
    _check(binding, dtype, [90, 90], [1, 1], 4, 2, 64, 16, scale=0.0)


@pytest.mark.parametrize("dtype", ALL, ids=list(ref.DTYPES))
@pytest.mark.parametrize("new", [1, 40])
def test_what_no_row_sees_gets_nothing(binding, dtype, new):
    # keys that are no numbers outside the window, infinite values inside it: weights do not depend on values
    lens = [200, 131]
    c = ref.cache(5, dtype, lens, [new, new], 2, 64, 16)
    for b in range(2):
        for j in range(3, lens[b] - new - 25):
            p, s = int(c["table"][b, j // 16]), j % 16
            c["k_pool"][p, :, s] = math.nan
            c["v_pool"][p, :, s] = math.inf
        p, s = int(c["table"][b, (lens[b] - 1) // 16]), (lens[b] - 1) % 16
        c["v_pool"][p, :, s, 3] = math.inf
    q = torch.randn((2 * new, 4, 64), generator=torch.Generator().manual_seed(1)).to(dtype)
    clean = {**c, "k_pool": c["k_pool"].nan_to_num(nan=0.0), "v_pool": torch.zeros_like(c["v_pool"])}
    sums, off = ref.mass(clean, q, 20, 3)
    before = torch.rand((2, 200))
    out, mass, status = _call(binding, c, q, before, 20, 3)
    assert status == [0, 0]
    assert torch.all((mass.double() - before.double() - sums).abs() <= off + ref.U32 * (before + sums))
    assert torch.equal(mass[sums == 0], before[sums == 0])


@pytest.mark.parametrize("dtype", ALL, ids=list(ref.DTYPES))
@pytest.mark.parametrize("new", [1, 30])
def test_bad_sequences_and_pages(binding, dtype, new):
    # sequence 1 has a page that is none, 2 is too long, 3 has more rows than tokens, 4 has none that are new
    lens, news = [70, 70, 90, new - 1 if new > 1 else 0, 33], [new, new, new, new, 0]
    c = ref.cache(3, dtype, lens, news, 2, 64, 16)
    q = torch.randn((c["T"], 4, 64), generator=torch.Generator().manual_seed(2)).to(dtype)
    sums, off = ref.mass(c, q)
    c["table"][1, 1] = 99
    before = torch.rand((5, 90))
    out, mass, status = _call(binding, c, q, before, max_len=80)
    assert status[0] == 0 and status[1] == 2 and status[2] == 1 and status[3:] == [0, 0]
    for b in (0, 3):
        assert torch.all((mass[b].double() - before[b].double() - sums[b]).abs() <= off[b] + ref.U32 * (before[b] + sums[b]))
    assert torch.equal(mass[2], before[2]) and torch.equal(mass[4], before[4])
    assert torch.isnan(mass[1, :70]).all() and torch.equal(mass[1, 70:], before[1, 70:])
    assert torch.all(out[2 * new:3 * new] == -3.0)
    # places that mass has no room for: the sequence is bad
    _, mass, status = _call(binding, c, q, before[:, :50].contiguous())
    assert status[0] == 1 and torch.equal(mass[0], before[0, :50])


@pytest.mark.parametrize("new", [1, 100])
def test_the_same_bits_with_any_stride_twice_and_in_a_graph(binding, new):
    c = ref.cache(9, torch.bfloat16, [700, 333], [new, new], 2, 128, 16)
    q = torch.randn((2 * new, 8, 128), generator=torch.Generator().manual_seed(4)).bfloat16()
    before = torch.rand((2, 800))
    out, mass, _ = _call(binding, c, q, before)
    again = _call(binding, c, q, before)
    assert torch.equal(out, again[0]) and torch.equal(mass, again[1])
    wide = torch.empty((2 * new, 8 * 128 + 5), dtype=torch.bfloat16, device=DEV)
    kp, vp, table, lens, starts = ref.on(DEV, c)
    for at in (0, 1):
        x = wide[:, at:at + 8 * 128].unflatten(1, (8, 128))
        x.copy_(q)
        m = before.to(DEV)
        got, _ = binding.approxifer_attend_mass(x, kp, vp, table, lens, starts, m, new, 700)
        assert torch.equal(m.cpu(), mass) and torch.equal(got.cpu(), out)
    ws = torch.empty((binding.approxifer_attend_mass_workspace_bytes(2 * new, 2, 8, 2, 128, torch.bfloat16, new, 700),), dtype=torch.uint8,
                     device=DEV)
    qd, m, o, st = q.to(DEV), before.to(DEV), torch.empty(q.shape, dtype=q.dtype, device=DEV), torch.empty((2,), dtype=torch.int32, device=DEV)
    side, graph = torch.cuda.Stream(), torch.cuda.CUDAGraph()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.graph(graph, stream=side):
        binding.approxifer_attend_mass(qd, kp, vp, table, lens, starts, m, new, 700, out=o, status=st, workspace=ws)
    for _ in range(3):
        m.copy_(before)
        o.zero_()
        ws.fill_(255)
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(m.cpu(), mass) and torch.equal(o.cpu(), out) and st.tolist() == [0, 0]
    m.copy_(before)
    torch.cuda.synchronize()
    o, _ = binding.approxifer_attend_mass(qd, kp, vp, table, lens, starts, m, new, 700, stream=side)
    side.synchronize()
    assert torch.equal(m.cpu(), mass) and torch.equal(o.cpu(), out)


def test_layers_add_up_and_attention_is_attends(binding):
    c = ref.cache(2, torch.float16, [400, 90, 5], [1, 1, 1], 2, 64, 16)
    q = torch.randn((3, 4, 64), generator=torch.Generator().manual_seed(4)).half()
    out, mass, _ = _call(binding, c, q, torch.zeros((3, 400)))
    sums, off = ref.mass(c, q)
    twice = _call(binding, c, q, mass)[1]
    assert torch.all((twice.double() - 2 * sums).abs() <= 2 * off + 3 * ref.U32 * sums)
    assert torch.all((mass.double().sum(1) - 4.0).abs() <= off.sum(1))           # the weights of four heads
    kp, vp, table, lens, starts = ref.on(DEV, c)
    plain, _ = binding.approxifer_attend(q.to(DEV), kp, vp, table, lens, starts, 1, 400)
    assert torch.equal(plain.cpu(), out)


def test_nothing_to_do_and_refusals(binding):
    c = ref.cache(2, torch.float16, [40, 9], [0, 0], 2, 64, 16)
    kp, vp, table, lens, starts = ref.on(DEV, c)
    mass = torch.ones((2, 40), device=DEV)
    none = torch.empty((0, 4, 64), dtype=torch.float16, device=DEV)
    _, status = binding.approxifer_attend_mass(none, kp, vp, table, lens, starts, mass, 1, 40, workspace=binding.NO_WORKSPACE)
    assert status.tolist() == [0, 0] and torch.all(mass == 1.0)
    q = torch.zeros((2, 4, 64), dtype=torch.float16, device=DEV)
    starts = torch.tensor([0, 1, 2], dtype=torch.int32, device=DEV)
    ws = _least(binding, 2, 4)
    for bad in (mass.half(), mass[0], mass[:1], mass.cpu(), mass.t()):
        with pytest.raises((TypeError, ValueError)):
            binding.approxifer_attend_mass(q, kp, vp, table, lens, starts, bad, 1, 40, workspace=ws)
    for small in (binding.NO_WORKSPACE, ws[:192]):
        with pytest.raises(binding.ApproxiferError) as e:
            binding.approxifer_attend_mass(q, kp, vp, table, lens, starts, mass, 1, 40, workspace=small)
        assert e.value.code == -12
    assert torch.all(mass == 1.0)


@pytest.mark.parametrize("dtype", ALL, ids=list(ref.DTYPES))
@pytest.mark.parametrize("heads,kv,dim", [(4, 1, 72), (2, 2, 96), (4, 2, 128), (3, 1, 200), (2, 1, 256)])
def test_prompts_on_either_side_of_what_keeps_its_scores(binding, dtype, heads, kv, dim):
    _check(binding, dtype, [256, 130, 41], [256, 130, 1], heads, kv, dim, 16)
    _check(binding, dtype, [400, 256, 3], [200, 17, 3], heads, kv, dim, 8, window=70, sinks=5)
    _check(binding, dtype, [300, 258, 257], [257, 258, 16], heads, kv, dim, 16)
