"""approxifer_attend for ragged batches of many sequences: which sequence a workgroup or a joining wave works for is looked up among
64 at a time, so batches of more than 64, 4096 and with runs of sequences without new tokens take every step of the search."""
import pytest
import torch

import sequence_reference as ref

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


def _check(dtype, lens, new, heads, kv, dim, window=0, sinks=0):
    from paper_2109_09868_amd import binding
    c = ref.cache(3, dtype, lens, new, kv, dim, 16)
    q = torch.randn((c["T"], heads, dim), generator=torch.Generator().manual_seed(4)).to(dtype)
    want, bound = ref.attend(c, q, window, sinks)
    x = q.to(DEV)
    for workspace in (None, binding.NO_WORKSPACE):
        out = torch.full(q.shape, -3.0, dtype=dtype, device=DEV)
        got, status = binding.approxifer_attend(x, *ref.on(DEV, c), max(new), max(lens), window=window, sinks=sinks, out=out,
                                                workspace=workspace)
        assert not status.any()
        off = (got.cpu().double() - want).abs()
        assert torch.all(off <= bound), (float(off.max()), int((off > bound).any(2).any(1).nonzero()[0]))


def _ragged(B, longest, kind):
    """Lengths and new tokens of B sequences: one of `longest`, some short ones, and runs without any."""
    lens = [1 + (7 * b) % 23 for b in range(B)]
    new = [(b % 3 if kind == "mixed" else int(b % 17 == 3)) if b % 5 or kind == "mixed" else 0 for b in range(B)]
    if kind in ("first", "last"):
        new = [0] * B
    at = {"mixed": B // 2, "runs": B - 1, "first": 0, "last": B - 1}[kind]
    lens[at] = new[at] = longest
    return lens, [min(n, l) for n, l in zip(new, lens)]


@pytest.mark.parametrize("dtype", list(ref.DTYPES.values()), ids=list(ref.DTYPES))
@pytest.mark.parametrize("kind", ["mixed", "runs", "first", "last"])
@pytest.mark.parametrize("B", [1, 2, 63, 64, 65, 130, 700])
def test_ragged_batches(dtype, kind, B):
    # a group of 3 heads: rows of a sequence begin and end inside the 128 of a workgroup
    lens, new = _ragged(B, 150, kind)
    _check(dtype, lens, new, 3, 1, 8)


@pytest.mark.parametrize("B", [4095, 4096, 4097, 5000])
def test_batches_that_take_three_steps(B):
    lens, new = _ragged(B, 131, "runs")
    _check(torch.bfloat16, lens, new, 1, 1, 8)


@pytest.mark.parametrize("dtype", [torch.float16, torch.bfloat16], ids=["f16", "bf16"])
def test_ragged_batches_whose_keys_are_cut(dtype):
    # more than 1024 rows in a few parts, and in many: one wave joins a row
    from paper_2109_09868_amd import binding
    for lens, new, least, most in (([2000], [1000], 2, 8), ([2000, 3, 700, 40], [990, 0, 1, 2], 2, 8), ([6000], [300], 9, 64)):
        T, B = sum(new), len(lens)
        need = binding.approxifer_attend_workspace_bytes(T, B, 4, 1, 64, dtype, max(new), max(lens))
        parts = need / ((T * 4 // 128 + B) * (128 * 64 + 256) * 4)
        assert parts == int(parts) and least <= parts <= most
        _check(dtype, lens, new, 4, 1, 64)
    _check(dtype, [3000, 3, 700, 40], [1000, 0, 1, 2], 4, 1, 64, window=1500, sinks=5)
