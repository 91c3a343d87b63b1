"""Sequences that have more of their own than max_len - max_shared says: in no group, in one that shares less, or in one that is refused.  Their keys are
cut as well, and parts that are empty are not looked at."""
import pytest
import torch

import sequence_reference as ref
from paper_2109_09868_amd import binding
from test_attend_shared import ALL, DEV, _cache, _call, _query


def _need(c, heads, kv, dim, dtype, C, new, max_shared, window=0, sinks=0):
    return binding.approxifer_attend_shared_workspace_bytes(c["T"], len(c["lens"]), C, heads, kv, dim, dtype, new, int(c["lens"].max()), max_shared,
                                                            window, sinks)


def test_parts_of_own_keys_are_planned():
    import os
    if not os.path.exists(binding.LIB_PATH):
        import __graft_entry__
        __graft_entry__.build()
    # float32, 12 heads of 64, behind 699 places: sequences of 700, and of which one may have many more of its own
    def parts(T, length):
        need, each = binding.approxifer_attend_shared_workspace_bytes(T, T, 1, 12, 12, 64, torch.float32, 1, length, 699), T * 12 * 66 * 4
        assert need % each == 0
        return need // each

    for T, length, own in ((24, 8000, 3), (30, 8000, 2), (24, 1600, 2), (8, 8000, 10), (600, 8000, 1)):
        assert parts(T, length) - parts(T, 700) >= own - 1, (T, length)
    # windows reach no more of them
    windowed = [binding.approxifer_attend_shared_workspace_bytes(24, 24, 1, 12, 12, 64, torch.float32, 1, n, 100, 500, 4) for n in (4000, 400000)]
    assert windowed[0] == windowed[1]


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ALL, ids=list(ref.DTYPES))
@pytest.mark.parametrize("heads,kv,dim,page", [(4, 4, 64, 16), (8, 2, 128, 16), (3, 3, 96, 8), (2, 1, 256, 64)])
def test_long_own_sequences_beside_a_group(dtype, heads, kv, dim, page):
    # a group of six behind 1800 places, one of two behind 40, two sequences in none: of 2500 and of 3; then the first group is refused
    own = [1, 30, 7, 800, 64, 65, 2300, 9, 2500, 3]
    groups, shared = [0, 6, 8], [1800, 40]
    c = _cache(3, dtype, groups, shared, own, [1] * 10, kv, dim, page)
    q = _query(c, heads, dim, dtype)
    for window, sinks in ((0, 0), (900, 5), (70, 2000)):
        want, bound = ref.attend(c, q, window, sinks)
        need = _need(c, heads, kv, dim, dtype, 2, 1, 1800, window, sinks)
        assert need % (10 * heads * (dim + 2) * 4) == 0
        for lengths in (shared, [1801, 40], [-1, 40]):
            got = []
            for _ in range(2):
                space = torch.full((need,), 255, dtype=torch.uint8, device=DEV)               # NaN wherever it is not written
                out, status = _call(binding, c, q, groups, lengths, window, sinks, workspace=space, max_shared=1800)
                assert status == [0] * 10 and torch.all((out.double() - want).abs() <= bound), (window, lengths)
                got.append(out)
            assert torch.equal(*got)


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ALL, ids=list(ref.DTYPES))
def test_rows_of_tiles_without_keys_in_a_part(dtype):
    # 160 rows of a group and head: tiles; windows that see nothing of what is common, and first tokens that do
    B = 20
    c = _cache(4, dtype, [0, B], [700], [5 + 9 * b for b in range(B)], [2] * B, 2, 64, 16)
    q = _query(c, 8, 64, dtype)
    for window, sinks in ((3, 0), (100, 0), (3, 10), (0, 0)):
        want, bound = ref.attend(c, q, window, sinks)
        need = _need(c, 8, 2, 64, dtype, 1, 2, 700, window, sinks)
        space = torch.full((need,), 255, dtype=torch.uint8, device=DEV)
        out, status = _call(binding, c, q, [0, B], [700], window, sinks, workspace=space)
        assert status == [0] * B and torch.all((out.double() - want).abs() <= bound), window
