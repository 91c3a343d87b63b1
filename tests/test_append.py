"""approxifer_append against the formulas in 64 bits."""
import numpy as np
import pytest
import torch

import sequence_reference as ref

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


@pytest.fixture(scope="module", params=["compiled", "ctypes"])
def binding(request):
    from paper_2109_09868_amd import binding
    binding.load()
    if request.param == "compiled":
        yield binding
        return
    patch = pytest.MonkeyPatch()
    patch.setattr(binding, "_marshal", lambda: (None, None))
    yield binding
    patch.undo()


def _run(binding, dtype, lens, new, heads, kv, dim, page, pairs, seed=0, interleaved=False, norm=True, axes=0, layout="fused",
         base=10000.0, places=None):
    c = ref.cache(seed, dtype, lens, new, kv, dim, page)
    g = torch.Generator().manual_seed(seed + 100)
    T = c["T"]
    rows = torch.randn((T, heads + 2 * kv, dim), generator=g).to(dtype)
    q, k, v = rows[:, :heads], rows[:, heads:heads + kv], rows[:, heads + kv:]
    qw, kw = (1 + 0.2 * torch.randn((2, dim), generator=g)).to(dtype) if norm else (None, None)
    freq = binding.approxifer_rotary_frequencies(pairs, base) if pairs else np.empty(0)
    positions = axis = None
    if axes:
        positions = torch.randint(-5, 900, (T, axes), generator=g, dtype=torch.int32)
        axis = np.arange(pairs, dtype=np.int32) * axes // max(pairs, 1)
    if places is not None:
        positions = torch.tensor(places, dtype=torch.int32)[:, None]
    want = ref.append(c, q, k, v, freq, qw, kw, 1e-6, positions, axis, interleaved)
    if layout == "fused":
        r = rows.to(DEV)
        q, k, v = r[:, :heads], r[:, heads:heads + kv], r[:, heads + kv:]
    elif layout == "odd":                                     # rows that begin at any element
        r = torch.empty((T, (heads + 2 * kv) * dim + 3), dtype=dtype, device=DEV)
        r[:, 1:-2] = rows.to(DEV).flatten(1)
        q, k, v = (r[:, a:a + n * dim].unflatten(1, (n, dim)) for a, n in
                   ((1, heads), (1 + heads * dim, kv), (1 + (heads + kv) * dim, kv)))
    else:
        q, k, v = (x.contiguous().to(DEV) for x in (q, k, v))
    kp, vp, table, lens_, starts = ref.on(DEV, c)
    qw, kw = (qw.to(DEV), kw.to(DEV)) if norm else (None, None)
    out = q if layout == "in place" else torch.full((T, heads, dim), -3.0, dtype=dtype, device=DEV)
    got, status = binding.approxifer_append(q, k, v, kp, vp, table, lens_, starts, freq, q_weight=qw, k_weight=kw,
                                            positions=positions.to(DEV) if positions is not None else None, axis=axis,
                                            interleaved=interleaved, q_out=out,
                                            status=torch.full((len(lens),), -1, dtype=torch.int32, device=DEV))
    assert got is out and torch.all(status == 0)
    for name, x, y, b in (("q", got, want[0], want[1]), ("k", kp, want[2], want[3]), ("v", vp, want[4], 0.0)):
        x = x.cpu().double()
        assert torch.equal(x.isnan(), y.isnan()), name
        off = (x - y).abs().nan_to_num(0.0)
        assert torch.all(off <= (b + 1e-30 if torch.is_tensor(b) else 0.0)), (name, float(off.max()))


@pytest.mark.parametrize("dtype", list(ref.DTYPES.values()), ids=list(ref.DTYPES))
@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("heads,kv,dim,pairs,page", [(12, 12, 64, 32, 16), (8, 2, 128, 64, 16), (6, 3, 80, 40, 8), (5, 1, 72, 36, 32),
                                                     (4, 4, 256, 64, 64), (2, 1, 8, 4, 1), (3, 3, 24, 5, 4), (16, 8, 128, 63, 16),
                                                     (33, 11, 40, 20, 128)])
def test_types_heads_and_layouts(binding, dtype, interleaved, heads, kv, dim, pairs, page):
    lens, new = [1, 7, 40, 33], [1, 2, 40, 0]
    for layout in ("fused", "plain", "odd", "in place"):
        _run(binding, dtype, lens, new, heads, kv, dim, page, pairs, interleaved=interleaved, layout=layout)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16], ids=["f32", "bf16"])
@pytest.mark.parametrize("axes", [1, 2, 3, 4])
def test_axes(binding, dtype, axes):
    for interleaved in (False, True):
        _run(binding, dtype, [37, 5], [37, 3], 4, 2, 96, 16, 48, interleaved=interleaved, norm=False, axes=axes)
        _run(binding, dtype, [37, 5], [37, 3], 4, 2, 96, 16, 17, interleaved=interleaved, axes=axes)


def test_without_rotation_and_without_norm(binding):
    for norm in (False, True):
        _run(binding, torch.float16, [3, 20], [3, 1], 4, 4, 64, 16, 0, norm=norm)
    _run(binding, torch.float32, [3, 20], [3, 1], 4, 4, 64, 16, 32, norm=False)


@pytest.mark.parametrize("interleaved", [False, True])
def test_far_positions(binding, interleaved):
    # angles of a million radians and more: a float32 product would be off by a tenth
    places = [0, 1, 131071, 1000003, 16777217, -1000003, 2 ** 30 + 1, 12345677]
    _run(binding, torch.float32, [8], [8], 2, 2, 64, 16, 32, places=places, interleaved=interleaved)


@pytest.mark.parametrize("T", [1, 2, 63, 64, 65, 1025])
def test_row_counts(binding, T):
    _run(binding, torch.bfloat16, [T + 3], [T], 4, 1, 64, 16, 32)


def test_many_sequences_of_few_tokens(binding):
    lens = [1 + (7 * b) % 50 for b in range(300)]
    _run(binding, torch.float16, lens, [min(l, b % 3) for b, l in enumerate(lens)], 2, 1, 32, 8, 16)


def test_extreme_values(binding):
    # norms of tiny and large rows; a zero row stays zero
    c = ref.cache(0, torch.float32, [3], [3], 1, 64, 16)
    g = torch.Generator().manual_seed(1)
    q = torch.randn((3, 1, 64), generator=g) * torch.tensor([1e-15, 1e15, 0.0])[:, None, None]
    w = torch.ones(64)
    want = ref.append(c, q, q, q, np.array([1.0]), w, w, 1e-6)
    kp, vp, table, lens, starts = ref.on(DEV, c)
    x = q.to(DEV)
    got, _ = binding.approxifer_append(x, x, x, kp, vp, table, lens, starts, np.array([1.0]), q_weight=w.to(DEV),
                                       k_weight=w.to(DEV))
    assert torch.all((got.cpu().double() - want[0]).abs() <= want[1])
    assert torch.all(got[2] == 0)


def test_bad_sequences_and_pages_are_told_and_harm_nobody(binding):
    lens, new = [20, 20, 20, 20, 20, 20], [4, 4, 4, 4, 4, 4]
    c = ref.cache(3, torch.float32, lens, new, 2, 64, 16)
    P = c["k_pool"].shape[0]
    c["table"][1, 1] = P                                      # the new tokens' page
    c["table"][2, 0] = -1                                     # a page that holds no new token: not needed
    c["lens"][3] = 33 * 16                                    # longer than the table
    c["table"][4, 1] = -2 ** 31
    c["lens"][5] = 2                                          # more new tokens than the length: two have no place
    g = torch.Generator().manual_seed(4)
    q, k = torch.randn((24, 4, 64), generator=g), torch.randn((24, 2, 64), generator=g)
    freq = binding.approxifer_rotary_frequencies(32)
    kp, vp, table, lens_, starts = ref.on(DEV, c)
    out = torch.full((24, 4, 64), -3.0, device=DEV)
    _, status = binding.approxifer_append(q.to(DEV), k.to(DEV), k.to(DEV), kp, vp, table, lens_, starts, freq, q_out=out,
                                          status=torch.full((6,), -1, dtype=torch.int32, device=DEV))
    assert status.tolist() == [0, 2, 0, 1, 2, 0]
    assert torch.all(out[12:16] == -3.0) and not torch.any(out[:12] == -3.0) and not torch.any(out[16:] == -3.0)
    good = {**c, "k_pool": c["k_pool"].clone(), "v_pool": c["v_pool"].clone()}
    for b in (1, 3, 4):                                       # the others are written
        good["lens"] = good["lens"].clone()
        good["lens"][b] = 0
    good["table"] = c["table"].clamp(0, P - 1)
    want = ref.append(good, q, k, k, freq)
    assert torch.equal(vp.cpu().double().nan_to_num(9.0), want[4].nan_to_num(9.0))
    # rows outside the T that there are, and in the wrong order
    starts = torch.tensor([0, 4, 30, 12, 16, 20, 24], dtype=torch.int32, device=DEV)
    _, status = binding.approxifer_append(q.to(DEV), k.to(DEV), k.to(DEV), kp, vp, table, lens_, starts, freq, q_out=out,
                                          status=status)
    assert status.tolist()[:3] == [0, 1, 1]


def test_no_rows(binding):
    c = ref.cache(0, torch.float32, [5, 0], [0, 0], 2, 64, 16)
    kp, vp, table, lens, starts = ref.on(DEV, c)
    q, k = torch.empty((0, 4, 64), device=DEV), torch.empty((0, 2, 64), device=DEV)
    out, status = binding.approxifer_append(q, k, k, kp, vp, table, lens, starts, binding.approxifer_rotary_frequencies(32))
    assert out.shape == (0, 4, 64) and status.tolist() == [0, 0]


def test_graph_replays_and_other_streams(binding):
    c = ref.cache(0, torch.float16, [9, 30], [9, 5], 2, 64, 16)
    g = torch.Generator().manual_seed(4)
    q, k = torch.randn((14, 4, 64), generator=g).half(), torch.randn((14, 2, 64), generator=g).half()
    freq = binding.approxifer_rotary_frequencies(32)
    want = ref.append(c, q, k, k, freq)
    kp, vp, table, lens, starts = ref.on(DEV, c)
    q, k = q.to(DEV), k.to(DEV)
    out, status = torch.empty_like(q), torch.empty((2,), dtype=torch.int32, device=DEV)
    side = torch.cuda.Stream()
    graph = torch.cuda.CUDAGraph()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.graph(graph, stream=side):
        binding.approxifer_append(q, k, k, kp, vp, table, lens, starts, freq, q_out=out, status=status)
    for _ in range(4):
        out.fill_(7.0)
        status.fill_(-1)
        graph.replay()
        torch.cuda.synchronize()
        assert torch.all((out.cpu().double() - want[0]).abs() <= want[1]) and status.tolist() == [0, 0]


@pytest.mark.parametrize("interleaved", [True, 1, np.True_, np.int64(3), False, 0, np.False_, None], ids=repr)
def test_what_counts_as_interleaved(binding, interleaved):
    _run(binding, torch.bfloat16, [20, 3], [20, 1], 4, 2, 64, 16, 32, interleaved=interleaved)
