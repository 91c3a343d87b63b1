"""A cache that weighs says that it does not read together what is shared."""
import warnings

import pytest


@pytest.fixture(params=["references", pytest.param("library", marks=pytest.mark.gpu)])
def device(request):
    import torch
    return torch.device("cpu" if request.param == "references" else "cuda:0")


@pytest.mark.parametrize("weigh", [False, True])
def test_a_word_where_both_are_asked_for(device, weigh):
    import os

    from paper_2109_09868_amd import binding, sequences
    if not os.path.exists(binding.LIB_PATH):
        import __graft_entry__
        __graft_entry__.build()
    cache = sequences.SequenceCache(1, 2, 2, 16, 4, 4, 20, device, weigh=weigh)
    cache.begin(4)
    with warnings.catch_warnings(record=True) as got:
        warnings.simplefilter("always")
        cache.share([0, 4], [3])
    assert [w.category for w in got] == [UserWarning] * weigh
